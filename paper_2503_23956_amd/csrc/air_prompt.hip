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
#include <math.h>
#include <string.h>

#include "air_device.h"
#include "air_internal.h"
#include "air_tile.h"

namespace air {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

struct PromptSpan {
    int64_t q_off, k_off, v_off, out_off;
    int32_t q_len, kv_len;
};
struct PromptArgs {
    const void *q, *k, *v;
    void *out;
    float *part_o;    // [split][KV head][row][D]
    float2 *part_ml;  // [split][KV head][row]
    int64_t q_h, q_t, k_h, k_t, v_h, v_t, out_h, out_t;
    float c;  // scale * log2(e)
    int32_t G, Hkv, n_seqs, n_tiles, n_rows, splits;
    int32_t tile0[AIR_MAX_BATCH];  // first row tile of a sequence in the launch; behind the last sequence: INT32_MAX
    int32_t row0[AIR_MAX_BATCH];   // first row (query x query head of the group) in the partial results, likewise
    PromptSpan s[AIR_MAX_BATCH];
};
static_assert(AIR_MAX_BATCH == 64 && sizeof(PromptArgs) <= 4096, "one lane per sequence; the size of an argument block");

// the last sequence whose first tile (row) is not behind x: one load for all sequences, not a chain of them
__device__ __forceinline__ int sequence_of(const int32_t *first, int x) {
    return __popcll(__ballot(first[threadIdx.x & 63] <= x)) - 1;
}

// What the wave functions need of the storage type: CH 16-byte pieces of a row, slices of 32 bytes (one piece per lane half)
template <typename T, int D>
struct Row {
    static constexpr int kVec = Elem<T>::kVec, kPieces = D / kVec, kSlices = kPieces / 2;
    // Where piece p of key r lies in its tile (64 banks of 4 bytes: 256 bytes of a tile are read at a time).
    // K: 16 bytes a lane, a row per lane: 16 neighbouring rows' pieces p lie in different banks.  V in bf16: read transposed, 32 lanes take
    // four rows x two neighbouring pairs of pieces: eight different pairs; in fp32 half a wave takes 128 bytes of row r, the
    // other half those of row r + 4.
    static __device__ __forceinline__ int k_at(int r, int p) { return r * kPieces + (p ^ (kPieces == 8 ? (r >> 1) & 7 : r & 15)); }
    static __device__ __forceinline__ int v_at(int r, int p) {
        if (sizeof(T) == 4) return r * kPieces + (p ^ ((r & 4) << 1));
        return r * kPieces + (p ^ (kPieces == 8 ? (r & 2) << 1 : ((r & 3) << 2) | ((r & 4) >> 1)));
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

// all exponent bits set in one of the elements
__device__ __forceinline__ bool not_finite(const uint4 &x, bf16_t) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad = bad || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}
__device__ __forceinline__ bool not_finite(const uint4 &x, float) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad = bad || (w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}

// the elements that are finite, 0 in place of the others
__device__ __forceinline__ u32x4 finite_part(u32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = (x[i] & 0x7f80u) == 0x7f80u ? 0u : x[i] & 0xffffu;
        const uint32_t hi = (x[i] & 0x7f800000u) == 0x7f800000u ? 0u : x[i] & 0xffff0000u;
        x[i] = lo | hi;
    }
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
// orders the LDS accesses of the lanes of one wave
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// s * c rounded, less the reference (two operations, not one)
__device__ __forceinline__ float rounded_exponent(float s, float c, float ref) {
#pragma clang fp contract(off)
    const float x = s * c;
    return x - ref;
}

constexpr float kHuge = 0x1p26f;
constexpr float kSlack = 8.0f;  // probabilities may be as large as 2^8: fp32 sums and bf16 operands hold them without loss

// RT row tiles of 32 of one wave against KT key tiles of 32 in LDS
template <typename T, int D, int RT, int KT>
struct Attend {
    using R = Row<T, D>;
    static constexpr int ND = D / 32;  // output tiles of 32 columns
    f32x16 acc[RT][ND];
    float m[RT], l[RT];  // reference (scaled logits), this lane's part of the sum
    uint4 q[RT][R::kSlices];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[r][d][i] = 0.f;
        }
    }

    // kb: first key of the tile in the sequence; last[r]: last key that the lane's query of row tile r sees (read when MASKED);
    // by_hand: the tile has values that are not finite at keys that some row does not see
    template <bool MASKED>
    __device__ __forceinline__ void step(const uint4 *sk, const uint4 *sv, int kb, const int (&last)[RT], float c, bool by_hand,
                                         float *scratch) {
        const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
        f32x16 s[RT][KT];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[r][kt][i] = 0.f;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const uint4 a = sk[R::k_at(32 * kt + n, 2 * sl + h)];
#pragma unroll
                for (int r = 0; r < RT; ++r) s[r][kt] = mma32(a, q[r][sl], s[r][kt], T());
            }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (MASKED) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (kb + 32 * kt + 8 * (i >> 2) + 4 * h + (i & 3) > last[r]) s[r][kt][i] = -INFINITY;
            }
            float mx = s[r][0][0];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[r][kt][i]);
            mx *= c;
            if (__ballot(mx > m[r] + kSlack) != 0ull) {
                const float m_new = fmaxf(m[r], fmaxf(mx, __shfl_xor(mx, 32, 64)));
                const float f = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[r] - m_new);  // no logit but -inf yet: nothing to scale
                l[r] *= f;
                m[r] = m_new;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[r][d][i] *= f;
            }
            const float ref = m[r] == -INFINITY ? 0.f : m[r];
            // The reference is a rounded product, the exponent an exact one minus it: the largest logit's exponent is off zero by half a
            // step of the reference, the same for all keys of the row, so that it cancels.  Far beyond any trained model's logits that
            // step leaves fp32's range of exponents: there the product is rounded as the reference was.
            if (__ballot(fabsf(ref) > kHuge) == 0ull) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][kt][i] = __builtin_amdgcn_exp2f(fmaf(s[r][kt][i], c, -ref));
            } else {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][kt][i] = __builtin_amdgcn_exp2f(rounded_exponent(s[r][kt][i], c, ref));
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) l[r] += s[r][kt][i];
        }
        if (MASKED && by_hand) {  // (uniform over the wave) a product with 0 would be NaN: only what a row sees is added
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {  // 16 keys at a time
                        wave_sync();
#pragma unroll
                        for (int i = 0; i < 8; ++i) scratch[32 * (8 * (i >> 2) + 4 * h + (i & 3)) + n] = s[r][kt][8 * half + i];
                        wave_sync();
                        for (int j = 0; j < 16; ++j) {
                            const int key = 32 * kt + 16 * half + j;
                            const bool sees = kb + key <= last[r];
                            const float p = scratch[32 * j + n];
                            const T *row = reinterpret_cast<const T *>(sv);
#pragma unroll
                            for (int d = 0; d < ND; ++d)
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const int col = 32 * d + 8 * (i >> 2) + 4 * h + (i & 3);
                                    const float v = ldf(row + R::v_at(key, col / R::kVec) * R::kVec + col % R::kVec);
                                    acc[r][d][i] = sees ? fmaf(p, v, acc[r][d][i]) : acc[r][d][i];
                                }
                        }
                    }
                }
            return;
        }
        if constexpr (sizeof(T) == 2) {
            // lane of the transposed read: row (lane % 16) / 4 of four keys, 8 bytes at columns 16 ((lane / 16) % 2) + 4 (lane % 4)
            const int krow = 4 * h + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const char *base = reinterpret_cast<const char *>(sv) + 8 * (lane & 1);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint4 p[RT];
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        bf16x8 x;
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = (__bf16)s[r][kt][8 * half + i];
                        p[r] = __builtin_bit_cast(uint4, x);
                    }
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const char *at = base + 16 * R::v_at(32 * kt + 16 * half + krow, 4 * d + piece);
                        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                        struct { s16x4 a, b; } v;
                        v.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
                        v.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * D * sizeof(T)));
#pragma unroll
                        for (int r = 0; r < RT; ++r) acc[r][d] = mma32(__builtin_bit_cast(uint4, v), p[r], acc[r][d], T());
                    }
                }
        } else {
            const float *base = reinterpret_cast<const float *>(sv) + 4 * h * D;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const float v = base[(32 * kt + 8 * (i >> 2) + (i & 3)) * D + ((32 * d + n) ^ (32 * h))];
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            acc[r][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r][kt][i], acc[r][d], 0, 0, 0);
                    }
        }
    }
};

// four consecutive output elements
__device__ __forceinline__ void store4(bf16_t *p, const f32x4 &x) {
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
    bf16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<uint2 *>(p) = __builtin_bit_cast(uint2, v);
}
__device__ __forceinline__ void store4(float *p, const f32x4 &x) { *reinterpret_cast<f32x4 *>(p) = x; }

// sequence, row tile, KV head and split of a workgroup.  The KV head is the fastest index (with 1, 2, 4 or 8 of them every XCD, dealt
// workgroups round-robin, works on one head's K and V); the tiles come last to first: the ones with the most keys first.
struct Place {
    int seq, tile, kvh, split;
};
__device__ __forceinline__ Place place_of(const PromptArgs &a, int w) {
    Place p;
    int x = w / a.Hkv;
    p.kvh = w - x * a.Hkv;
    const int y = x / a.splits;
    p.split = x - y * a.splits;
    const int tile = a.n_tiles - 1 - y;
    p.seq = a.n_seqs == 1 ? 0 : sequence_of(a.tile0, tile);
    p.tile = tile - (a.n_seqs == 1 ? 0 : a.tile0[p.seq]);
    return p;
}

// ---------------------------------------------------------------------------------------
// Many rows: NW waves of 32 RT rows each over tiles of 32 KT keys in LDS, which all waves share.  The next tile's loads are in
// flight while the present one is multiplied.
// ---------------------------------------------------------------------------------------
template <typename T, int D, int NW, int RT, int KT>
__global__ __launch_bounds__(64 * NW) void prompt_kernel(PromptArgs a) {
    using R = Row<T, D>;
    constexpr int kRows = 32 * RT * NW, kKeys = 32 * KT, kThreads = 64 * NW;
    constexpr int kLoads = kKeys * R::kPieces / kThreads, kRowStep = kThreads / R::kPieces;
    static_assert(kLoads * kThreads == kKeys * R::kPieces && kRowStep >= 1, "whole rounds of loads");
    __shared__ uint4 sk[2][kKeys * R::kPieces], sv[2][kKeys * R::kPieces];
    __shared__ float scratch[NW][16 * 32];
    __shared__ int s_bad;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(a, blockIdx.x);
    const PromptSpan &sp = a.s[pl.seq];
    const int n_rows = sp.q_len * a.G, shift = sp.kv_len - sp.q_len;
    const int row0 = pl.tile * kRows;
    const int end_row = min(row0 + kRows, n_rows);
    // keys that every row of the tile sees, and that any does
    const int see_all = max(0, row0 / a.G + shift + 1), see_any = max(0, (end_row - 1) / a.G + shift + 1);
    const int n_blocks = (see_any + kKeys - 1) / kKeys, n_full = see_all / kKeys;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    Attend<T, D, RT, KT> at;
    at.clear();
    int last[RT], head[RT], tok[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + 32 * (RT * wave + r) + n, n_rows - 1);
        tok[r] = row / a.G;
        head[r] = pl.kvh * a.G + row - tok[r] * a.G;
        last[r] = tok[r] + shift;
        const T *q = (const T *)a.q + sp.q_off + tok[r] * a.q_t + head[r] * a.q_h;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl) at.q[r][sl] = *reinterpret_cast<const uint4 *>(q + R::kVec * (2 * sl + h));
    }

    const T *kg = (const T *)a.k + sp.k_off + pl.kvh * a.k_h, *vg = (const T *)a.v + sp.v_off + pl.kvh * a.v_h;
    const int piece = threadIdx.x % R::kPieces, lrow = threadIdx.x / R::kPieces;
    uint4 kr[kLoads], vr[kLoads];
    auto load = [&](int b) {
        const int kb = b * kKeys, top = sp.kv_len - 1 - kb;  // rows past the last key re-read it
        const T *kp = kg + kb * a.k_t + R::kVec * piece, *vp = vg + kb * a.v_t + R::kVec * piece;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = min(lrow + kRowStep * i, top);
            kr[i] = *reinterpret_cast<const uint4 *>(kp + r * a.k_t);
            vr[i] = *reinterpret_cast<const uint4 *>(vp + r * a.v_t);
        }
    };
    auto keep = [&](int b) {
        const int buf = b & 1;
        if (b >= n_full) {  // some row does not see all of the tile
            const int left = sp.kv_len - b * kKeys;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (lrow + kRowStep * i >= left) vr[i] = make_uint4(0, 0, 0, 0);
                bad = bad || not_finite(vr[i], T());
            }
            if (bad) s_bad = 1;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            sk[buf][R::k_at(lrow + kRowStep * i, piece)] = kr[i];
            sv[buf][R::v_at(lrow + kRowStep * i, piece)] = vr[i];
        }
    };
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    if (b0 < b1) {
        load(b0);
        keep(b0);
    }
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        if (b + 1 < b1) load(b + 1);
        if (b < n_full) at.template step<false>(sk[b & 1], sv[b & 1], b * kKeys, last, a.c, false, scratch[wave]);
        else at.template step<true>(sk[b & 1], sv[b & 1], b * kKeys, last, a.c, __builtin_amdgcn_readfirstlane(s_bad) != 0, scratch[wave]);
        if (b + 1 < b1) keep(b + 1);
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float l = at.l[r] + __shfl_xor(at.l[r], 32, 64);
        const int row = row0 + 32 * (RT * wave + r) + n;
        if (row >= n_rows) continue;
        if (a.splits == 1) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            T *o = (T *)a.out + sp.out_off + tok[r] * a.out_t + head[r] * a.out_h;
#pragma unroll
            for (int d = 0; d < Attend<T, D, RT, KT>::ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 x;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : at.acc[r][d][4 * i + j] * inv;
                    store4(o + 32 * d + 8 * i + 4 * h, x);
                }
        } else {
            const int64_t slot = ((int64_t)pl.split * a.Hkv + pl.kvh) * a.n_rows + a.row0[pl.seq] + row;
            if (h == 0) a.part_ml[slot] = make_float2(at.m[r], l);
            float *o = a.part_o + slot * D;
#pragma unroll
            for (int d = 0; d < Attend<T, D, RT, KT>::ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 x;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = at.acc[r][d][4 * i + j];
                    store4(o + 32 * d + 8 * i + 4 * h, x);
                }
        }
    }
}

// ---------------------------------------------------------------------------------------
// Many rows, bf16: 4 waves of 32 RT rows, key blocks of 64 in LDS (three buffers), two row tiles a wave so that what is read of
// K and V from LDS serves 64 rows.  One wave per SIMD: the logits of the next 32 keys are formed (matrix unit) while the
// exponentials of the present ones are (vector unit), in one run of instructions without a branch.
// ---------------------------------------------------------------------------------------
template <typename T, int D, int RT, int NW>
__global__ __launch_bounds__(64 * NW, NW / 4) void prompt_pipe_kernel(PromptArgs a) {
    using R = Row<T, D>;
    static_assert(sizeof(T) == 2, "bf16");
    constexpr int kRows = 32 * RT * NW, kKeys = 64, ND = D / 32, NS = R::kSlices, kBufs = 3;
    constexpr int kTile = kKeys * R::kPieces, kLoads = kTile / (64 * NW), kRowStep = 64 * NW / R::kPieces;
    __shared__ u32x4 sk[kBufs][kTile], sv[kBufs][kTile];
    __shared__ int s_bad;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(a, blockIdx.x);
    const PromptSpan &sp = a.s[pl.seq];
    const int n_rows = sp.q_len * a.G, shift = sp.kv_len - sp.q_len;
    const int row0 = pl.tile * kRows, end_row = min(row0 + kRows, n_rows);
    const int see_all = max(0, row0 / a.G + shift + 1), see_any = max(0, (end_row - 1) / a.G + shift + 1);
    const int n_blocks = (see_any + kKeys - 1) / kKeys;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    f32x16 acc[RT][ND];
    float l[RT], ref[RT], top[RT], mul[RT], sub[RT];  // top: the logit (scaled) from which on the reference is raised
    uint4 q[RT][NS];
    int last[RT], row[RT];
    bool huge = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        l[r] = 0.f;
        ref[r] = top[r] = -INFINITY;
        mul[r] = a.c;
        sub[r] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][d][i] = 0.f;
        row[r] = row0 + 32 * (RT * wave + r) + n;
        const int m = min(row[r], n_rows - 1), t = m / a.G, g = m - t * a.G;
        last[r] = t + shift;
        const T *qp = (const T *)a.q + sp.q_off + t * a.q_t + (pl.kvh * a.G + g) * a.q_h;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) q[r][sl] = *reinterpret_cast<const uint4 *>(qp + R::kVec * (2 * sl + h));
    }

    const T *kg = (const T *)a.k + sp.k_off + pl.kvh * a.k_h, *vg = (const T *)a.v + sp.v_off + pl.kvh * a.v_h;
    const int piece = threadIdx.x % R::kPieces, lrow = threadIdx.x / R::kPieces;
    const int64_t k_lane = lrow * a.k_t + R::kVec * piece, v_lane = lrow * a.v_t + R::kVec * piece;
    u32x4 kr[kLoads], vr[kLoads];
    auto load = [&](int b) {
        const int kb = b * kKeys, end = sp.kv_len - 1 - kb;
        const T *kp = kg + kb * a.k_t, *vp = vg + kb * a.v_t;
        if (end >= kKeys - 1) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                kr[i] = *reinterpret_cast<const u32x4 *>(kp + i * (kRowStep * a.k_t) + k_lane);
                vr[i] = *reinterpret_cast<const u32x4 *>(vp + i * (kRowStep * a.v_t) + v_lane);
            }
        } else {  // rows past the last key re-read it
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = min(lrow + kRowStep * i, end);
                kr[i] = *reinterpret_cast<const u32x4 *>(kp + r * a.k_t + R::kVec * piece);
                vr[i] = *reinterpret_cast<const u32x4 *>(vp + r * a.v_t + R::kVec * piece);
            }
        }
    };
    auto keep = [&](int b) {
        const int buf = b % kBufs;
        if ((b + 1) * kKeys > see_all) {
            // Some row does not see all of the block, and its probability of 0 must not meet an infinity: values behind the last key become
            // 0, and so does what is not finite (added at the end to the rows that see it)
            const int left = sp.kv_len - b * kKeys;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (lrow + kRowStep * i >= left) vr[i] = (u32x4){0, 0, 0, 0};
                if (not_finite(__builtin_bit_cast(uint4, vr[i]), T())) {
                    bad = true;
                    vr[i] = finite_part(vr[i]);
                }
            }
            if (bad) s_bad = 1;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            sk[buf][R::k_at(lrow + kRowStep * i, piece)] = kr[i];
            sv[buf][R::v_at(lrow + kRowStep * i, piece)] = vr[i];
        }
    };
    // operands of the logits of the 32 keys whose tile starts at sk_
    auto read_k = [&](u32x4(&x)[NS], const u32x4 *sk_) {
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) x[sl] = sk_[R::k_at(n, 2 * sl + h)];
    };
    auto largest = [&](const f32x16 &s) {
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        return mx;
    };
    auto logits = [&](f32x16(&s)[RT], const u32x4(&x)[NS]) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[r][i] = 0.f;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl)
#pragma unroll
            for (int r = 0; r < RT; ++r) s[r] = mma32(__builtin_bit_cast(uint4, x[sl]), q[r][sl], s[r], T());
    };
    // masks, reference: what has to be known of the logits of the keys from kb on before their exponentials are formed
    auto settle = [&](f32x16(&s)[RT], float(&mx)[RT], int kb) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (__builtin_expect(kb + 32 > see_all, 0)) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (kb + 8 * (i >> 2) + 4 * h + (i & 3) > last[r]) s[r][i] = -INFINITY;
                mx[r] = largest(s[r]);
            }
            mx[r] *= a.c;
            if (__builtin_expect(__ballot(mx[r] > top[r]) != 0ull, 0)) {
                const float now = fmaxf(ref[r], fmaxf(mx[r], __shfl_xor(mx[r], 32, 64)));
                const float f = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref[r] - now);  // no logit but -inf yet: nothing to scale
                l[r] *= f;
                ref[r] = now;
                top[r] = now + kSlack;
                sub[r] = now == -INFINITY ? 0.f : now;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[r][d][i] *= f;
                huge = huge || __ballot(fabsf(sub[r]) > kHuge) != 0ull;
            }
            if (__builtin_expect(huge, 0)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[r][i] = rounded_exponent(s[r][i], a.c, ref[r] == -INFINITY ? 0.f : ref[r]);
                mul[r] = 1.f;
                sub[r] = 0.f;
            }
        }
    };
    const int krow = 4 * h + ((lane & 15) >> 2), vpiece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    auto read_v = [&](u32x4(&x)[ND], const u32x4 *sv_, int half) {
        const char *base = reinterpret_cast<const char *>(sv_) + 8 * (lane & 1);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const char *at = base + 16 * R::v_at(16 * half + krow, 4 * d + vpiece);
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            struct { s16x4 a, b; } v;
            v.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
            v.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * D * sizeof(T)));
            x[d] = __builtin_bit_cast(u32x4, v);
        }
    };
    // The next 32 keys' logits into `next` (operands: kf) while this 32 keys' values are weighed; kf then takes the operands of the keys
    // behind those.  `meet`: the tiles that k_after points to are whole only behind a barrier.
    auto turn = [&](f32x16(&s)[RT], f32x16(&next)[RT], float(&mx)[RT], u32x4(&kf)[NS], const u32x4 *sv_, const u32x4 *k_after, bool meet) {
        u32x4 vf[2][ND];
        __builtin_amdgcn_s_setprio(1);
        read_v(vf[0], sv_, 0);
        logits(next, kf);
        uint4 p[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                bf16x8 x;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[r][8 * half + i], mul[r], -sub[r]));
                p[r][half] = __builtin_bit_cast(uint4, x);
            }
        read_v(vf[1], sv_, 1);
        if (meet) lds_barrier();
        read_k(kf, k_after);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[r][d] = mma32(__builtin_bit_cast(uint4, vf[half][d]), p[r][half], acc[r][d], T());
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            // the sum of what the second product takes: the weights add up to one as they are used
            l[r] = sum_of(p[r][1], sum_of(p[r][0], l[r]));
            mx[r] = largest(next[r]);
        }
        __builtin_amdgcn_s_setprio(0);
        if (!meet) {
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, RT, 0);
                __builtin_amdgcn_sched_group_barrier(0x2, 40 / NS, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }

#pragma unroll
            for (int i = 0; i < 2 * ND; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, RT, 0);
                __builtin_amdgcn_sched_group_barrier(0x2, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
        }
    };
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    if (b0 < b1) {
        f32x16 sa[RT], sb[RT];
        float mx[RT];
        u32x4 kf[NS];
        load(b0);
        keep(b0);
        if (b0 + 1 < b1) load(b0 + 1);
        lds_barrier();
        read_k(kf, sk[b0 % kBufs]);
        logits(sa, kf);
#pragma unroll
        for (int r = 0; r < RT; ++r) mx[r] = largest(sa[r]);
        settle(sa, mx, b0 * kKeys);
        read_k(kf, sk[b0 % kBufs] + 32 * R::kPieces);
        for (int b = b0; b < b1; ++b) {
            const u32x4 *v_now = sv[b % kBufs], *k_next = sk[(b + 1) % kBufs];
            if (b + 1 < b1) keep(b + 1);
            if (b + 2 < b1) load(b + 2);
            turn(sa, sb, mx, kf, v_now, k_next, true);
            settle(sb, mx, b * kKeys + 32);
            // (behind the last block: logits of whatever lies there, not used)
            turn(sb, sa, mx, kf, v_now + 32 * R::kPieces, k_next + 32 * R::kPieces, false);
            if (b + 1 < b1) settle(sa, mx, (b + 1) * kKeys);
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float sum = l[r] + __shfl_xor(l[r], 32, 64);
        if (row[r] >= n_rows) continue;
        if (s_bad) {  // values that are not finite, at keys that some row does not see
            for (int key = max(b0 * kKeys, see_all / kKeys * kKeys); key < min(b1 * kKeys, see_any); ++key) {
                if (key > last[r]) continue;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float v = ldf(vg + key * a.v_t + 32 * d + 8 * (i >> 2) + 4 * h + (i & 3));
                        if (!(fabsf(v) < INFINITY)) acc[r][d][i] += v;
                    }
            }
        }
        const int t = row[r] / a.G, head = pl.kvh * a.G + row[r] - t * a.G;
        const bool whole = a.splits == 1;
        const float inv = whole ? 1.0f / sum : 1.0f;
        const bool none = whole && sum == 0.f;
        const int64_t slot = ((int64_t)pl.split * a.Hkv + pl.kvh) * a.n_rows + a.row0[pl.seq] + row[r];
        if (!whole && h == 0) a.part_ml[slot] = make_float2(ref[r], sum);
        T *o = (T *)a.out + sp.out_off + t * a.out_t + head * a.out_h;
        float *po = a.part_o + slot * D;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = none ? 0.f : acc[r][d][4 * i + j] * inv;
                const int col = 32 * d + 8 * i + 4 * h;
                if (whole) store4(o + col, x);
                else store4(po + col, x);
            }
    }
}

// ---------------------------------------------------------------------------------------
// Few rows (at most 32 per KV head and sequence): bound by reading K and V.  Four waves share the rows and deal the key tiles of 32
// among themselves; each moves its tiles through LDS of its own, the next tile's loads in flight, without a barrier.
// ---------------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_few_kernel(PromptArgs a) {
    using R = Row<T, D>;
    constexpr int kTile = 32 * R::kPieces, kLoads = kTile / 64, kRowStep = 64 / R::kPieces, NW = 4;
    __shared__ uint4 tiles[NW][2][kTile];
    __shared__ float scratch[NW][16 * 32];
    __shared__ float s_m[NW][32], s_l[NW][32];
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(a, blockIdx.x);
    const PromptSpan &sp = a.s[pl.seq];
    const int n_rows = sp.q_len * a.G, shift = sp.kv_len - sp.q_len;
    const int row0 = pl.tile * 32, end_row = min(row0 + 32, n_rows);
    const int see_all = max(0, row0 / a.G + shift + 1), see_any = max(0, (end_row - 1) / a.G + shift + 1);
    const int n_blocks = (see_any + 31) / 32, n_full = see_all / 32;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    Attend<T, D, 1, 1> at;
    at.clear();
    const int row = min(row0 + n, n_rows - 1), tok = row / a.G, head = pl.kvh * a.G + row - tok * a.G;
    const int last[1] = {tok + shift};
    {
        const T *q = (const T *)a.q + sp.q_off + tok * a.q_t + head * a.q_h;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl) at.q[0][sl] = *reinterpret_cast<const uint4 *>(q + R::kVec * (2 * sl + h));
    }
    const T *kg = (const T *)a.k + sp.k_off + pl.kvh * a.k_h, *vg = (const T *)a.v + sp.v_off + pl.kvh * a.v_h;
    const int piece = lane % R::kPieces, lrow = lane / R::kPieces;
    uint4 *sk = tiles[wave][0], *sv = tiles[wave][1];
    uint4 kr[kLoads], vr[kLoads];
    auto load = [&](int b) {
        const int kb = b * 32, top = sp.kv_len - 1 - kb;
        const T *kp = kg + kb * a.k_t + R::kVec * piece, *vp = vg + kb * a.v_t + R::kVec * piece;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kp + min(lrow + kRowStep * i, top) * a.k_t);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) vr[i] = *reinterpret_cast<const uint4 *>(vp + min(lrow + kRowStep * i, top) * a.v_t);
    };
    int b = b0 + wave;
    if (b < b1) load(b);
    for (; b < b1; b += NW) {
        bool bad = false;
        if (b >= n_full) {
            const int left = sp.kv_len - b * 32;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (lrow + kRowStep * i >= left) vr[i] = make_uint4(0, 0, 0, 0);
                bad = bad || not_finite(vr[i], T());
            }
            bad = __ballot(bad) != 0ull;
        }
        wave_sync();  // the wave's reads of the tile before are behind it
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            sk[R::k_at(lrow + kRowStep * i, piece)] = kr[i];
            sv[R::v_at(lrow + kRowStep * i, piece)] = vr[i];
        }
        wave_sync();
        if (b + NW < b1) load(b + NW);
        if (b < n_full) at.template step<false>(sk, sv, b * 32, last, a.c, false, scratch[wave]);
        else at.template step<true>(sk, sv, b * 32, last, a.c, bad, scratch[wave]);
    }
    // merge of the four waves: every wave brings its sums to the common reference and leaves them in LDS
    const float l = at.l[0] + __shfl_xor(at.l[0], 32, 64);
    if (h == 0) s_m[wave][n] = at.m[0];
    __syncthreads();
    float M = s_m[0][n];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][n]);
    const float f = at.m[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(at.m[0] - M);
    if (h == 0) s_l[wave][n] = l * f;
    constexpr int kQuads = D / 4;  // 16-byte pieces of a row of sums
    static_assert(sizeof(tiles) >= NW * 32 * D * sizeof(float), "the tiles' memory holds the sums");
    f32x4 *sums = reinterpret_cast<f32x4 *>(&tiles[0][0][0]);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = f == 0.f ? 0.f : at.acc[0][d][4 * i + j] * f;
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
        const int t = (row0 + r) / a.G, g = row0 + r - t * a.G;
        if (a.splits == 1) {
            const float inv = 1.0f / lt;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = lt == 0.f ? 0.f : x[j] * inv;
            store4((T *)a.out + sp.out_off + t * a.out_t + (pl.kvh * a.G + g) * a.out_h + 4 * c4, x);
        } else {
            const int64_t slot = ((int64_t)pl.split * a.Hkv + pl.kvh) * a.n_rows + a.row0[pl.seq] + row0 + r;
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
template <typename T, int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, int groups) {
    constexpr int kQuads = D / 4, kRound = 8;
    __shared__ f32x4 s_x[256];
    __shared__ float2 s_ml[256 / kQuads];
    const int c4 = threadIdx.x % kQuads, team = threadIdx.x / kQuads, g = team & (groups - 1);
    const int64_t idx = (int64_t)blockIdx.x * (256 / kQuads / groups) + team / groups;
    const bool live = idx < (int64_t)a.n_rows * a.Hkv;
    const int64_t stride = (int64_t)a.Hkv * a.n_rows;
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
        if (top == -INFINITY) top = 0.f;
        const float f = __builtin_amdgcn_exp2f(m - top);
        l *= f;
        x *= f;
        m = top;
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            if (s0 + i * groups >= a.splits || ml[i].y == 0.f) continue;  // (a split that saw nothing left nothing)
            const float w = __builtin_amdgcn_exp2f(ml[i].x - m);
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
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l *= f;
        x *= f;
        for (int i = 1; i < groups; ++i) {
            const float2 ml = s_ml[team + i];
            if (ml.y == 0.f) continue;
            const float w = __builtin_amdgcn_exp2f(ml.x - top);
            l = fmaf(w, ml.y, l);
            const f32x4 o = s_x[threadIdx.x + i * kQuads];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(w, o[j], x[j]);
        }
    }
    if (!live) return;
    const int kvh = (int)(idx / a.n_rows), row = (int)(idx - (int64_t)kvh * a.n_rows);
    int seq = 0;  // (lanes differ in their row: no vote here)
    for (int step = 32; step > 0; step >>= 1)
        if (a.row0[seq + step] <= row) seq += step;
    const PromptSpan &sp = a.s[seq];
    const int r = row - a.row0[seq], t = r / a.G, q = r - t * a.G;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : x[j] / l;
    store4((T *)a.out + sp.out_off + t * a.out_t + (kvh * a.G + q) * a.out_h + 4 * c4, x);
}

// ---------------------------------------------------------------------------------------
// The shape of a call: which kernel, how many splits, what the partial results take
// ---------------------------------------------------------------------------------------
struct PromptPlan {
    bool few;
    int tile_rows, splits;
    int64_t n_tiles, n_rows;
    size_t ml_bytes, bytes;
};
static PromptPlan plan_of(const air_prompt_config &c, const air_prompt_seq *seqs, int n) {
    const int64_t G = c.n_q_heads / c.n_kv_heads;
    PromptPlan p;
    memset(&p, 0, sizeof(p));
    int64_t most = 0, keys = 0;
    for (int i = 0; i < n; ++i) {
        if (seqs[i].q_len * G > most) most = seqs[i].q_len * G;
        if (seqs[i].q_len > 0 && seqs[i].kv_len > keys) keys = seqs[i].kv_len;
    }
    p.few = most <= 32;
    p.tile_rows = p.few ? 32 : (c.dtype == AIR_BF16 ? 256 : 128);
    for (int i = 0; i < n; ++i) {
        p.n_tiles += (seqs[i].q_len * G + p.tile_rows - 1) / p.tile_rows;
        p.n_rows += seqs[i].q_len * G;
    }
    p.splits = 1;
    const int64_t wgs = p.n_tiles * c.n_kv_heads, per = p.few ? 128 : 512;
    if (wgs > 0) {
        while (p.splits < 64 && wgs * p.splits < kCUs && keys > p.splits * per) p.splits *= 2;
    }
    if (p.splits > 1) {
        const size_t slots = (size_t)p.n_rows * c.n_kv_heads * p.splits;
        p.ml_bytes = (slots * sizeof(float2) + 255) / 256 * 256;
        p.bytes = p.ml_bytes + slots * c.head_dim * sizeof(float);
    }
    return p;
}

size_t prompt_workspace(const air_prompt_config &c, const air_prompt_seq *seqs, int n) { return plan_of(c, seqs, n).bytes; }

bool prompt_grid_ok(const air_prompt_config &c, const air_prompt_seq *seqs, int n) {
    const PromptPlan p = plan_of(c, seqs, n);
    return p.n_rows * c.n_kv_heads < 0x7fffffffll / (c.head_dim / 4) && p.n_tiles * c.n_kv_heads * p.splits < 0x7fffffffll;
}

template <typename T, int D>
static void prompt_launch(hipStream_t s, const PromptPlan &p, const PromptArgs &a) {
    const dim3 grid((unsigned)(p.n_tiles * a.Hkv * p.splits));
    if (p.few) hipLaunchKernelGGL((prompt_few_kernel<T, D>), grid, dim3(256), 0, s, a);
    else if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((prompt_pipe_kernel<T, D, 1, 8>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((prompt_kernel<T, D, 4, 1, 1>), grid, dim3(256), 0, s, a);
    if (p.splits > 1) {
        constexpr int kMost = 256 / (D / 4);
        int groups = 1;
        while (groups < kMost && groups * 2 <= p.splits) groups *= 2;
        const int64_t per = kMost / groups, rows = p.n_rows * a.Hkv;
        hipLaunchKernelGGL((prompt_join_kernel<T, D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, s, a, groups);
    }
}

hipError_t launch_prompt(hipStream_t s, const air_prompt_config &c, const air_prompt_seq *seqs, int n, const void *q, const void *k,
                         const void *v, void *out, void *workspace) {
    const PromptPlan p = plan_of(c, seqs, n);
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
    a.c = (float)((c.scale > 0.f ? (double)c.scale : 1.0 / sqrt((double)c.head_dim)) * 1.4426950408889634);
    a.splits = p.splits;
    a.n_tiles = (int)p.n_tiles;
    a.n_rows = (int)p.n_rows;
    // sequences by rising length: the workgroups take the tiles from the last to the first, the longest first
    int order[AIR_MAX_BATCH];
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (seqs[i].q_len == 0) continue;
        int at = m++;
        for (; at > 0 && seqs[order[at - 1]].kv_len > seqs[i].kv_len; --at) order[at] = order[at - 1];
        order[at] = i;
    }
    a.n_seqs = m;
    int tile0 = 0, row0 = 0;
    for (int i = 0; i < AIR_MAX_BATCH; ++i) a.tile0[i] = a.row0[i] = 0x7fffffff;
    for (int i = 0; i < m; ++i) {
        const air_prompt_seq &x = seqs[order[i]];
        a.s[i] = PromptSpan{x.q_off, x.k_off, x.v_off, x.out_off, x.q_len, x.kv_len};
        a.tile0[i] = tile0;
        a.row0[i] = row0;
        const int rows = x.q_len * a.G;
        tile0 += (rows + p.tile_rows - 1) / p.tile_rows;
        row0 += rows;
    }
    if (c.dtype == AIR_BF16) c.head_dim == 128 ? prompt_launch<bf16_t, 128>(s, p, a) : prompt_launch<bf16_t, 64>(s, p, a);
    else c.head_dim == 128 ? prompt_launch<float, 128>(s, p, a) : prompt_launch<float, 64>(s, p, a);
    return hipGetLastError();
}

}  // namespace air
