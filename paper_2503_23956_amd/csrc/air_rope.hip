// air_rope: per-head RMS norm and position rotation of queries and keys, values laid out on the way.
//
// One read and one write of every element, bound by memory: a row (one token, one head) belongs to a group of
// head_dim / (2 kVec) lanes, a lane holds two 16-byte pieces that contain both halves of its pairs in either layout, so the
// rotation needs no exchange between lanes and the norm one sum over the group.  A group takes a run of heads of one token:
// the angles of its pairs (a chain of fp64 operations, a sine and a cosine each) are formed once for the run.
// 7432 tokens of 28 / 4 heads of 128 elements in bf16, values with them: 29 us, 4.7 TB/s (a plain copy 4.9); 32911 tokens of 64 / 8 heads with norms
// 292 us, 4.6 TB/s; one token 3.4 us in a graph, what any launch takes.
#include <math.h>
#include <string.h>

#include "air_device.h"
#include "air_internal.h"
#include "air_tile.h"

namespace air {

struct RopeArgs {
    air_rope_tensor t[3];
    int32_t heads[3], runs[3];  // heads of q, k, v (0: left out) and the runs of heads they are cut into
    int32_t n_tokens, rows;     // rows = batch * n_tokens
    int32_t n_axes, end0, end1, pairs;  // pairs [0, end0) turn with axis 0, [end0, end1) with axis 1, the rest with axis 2
    float eps, scale;
    const int32_t *positions;
    const double *freqs;
};

// 16 bytes to floats and back (one rounding)
__device__ __forceinline__ void unpack(const uint4 &x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4 &x, float (&f)[4]) {
    const f32x4 v = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = v[i];
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
    return __builtin_bit_cast(uint4, v);
}
__device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f[i];
    return __builtin_bit_cast(uint4, v);
}

// Cosine and sine of p f radians.  The product and 2 / pi are taken in two parts each, so that what is left when whole quarter turns are dropped
// is right to 2^-53 of a turn and 2^-100 of all turns: the same for positions of 2^31 as for small ones (in one part each, 2^-24 turns were
// lost there).  The rest z, rounded to fp32 once, is at most pi / 4: the series to z^9 and z^10 leave 2e-9 and 2e-10.
__device__ __forceinline__ void turn_by(double p, double f, float &cs, float &sn) {
#pragma clang fp contract(off)  // t less its quarters: of t as it was rounded, whose rest t_low holds
    constexpr double kHigh = 0x1.45f306dc9c883p-1, kLow = -0x1.6b01ec5417056p-55;  // 2 / pi
    const double x = p * f, x_low = fma(p, f, -x);
    const double t = x * kHigh, t_low = fma(x, kHigh, -t) + fma(x, kLow, x_low * kHigh);
    const double n = rint(t);
    const float z = (float)(((t - n) + t_low) * 1.5707963267948966), zz = z * z;
    const int k = __double2loint(n + 0x1.8p52);  // the quarters' last two bits
    const float s = fmaf(z * zz, fmaf(zz, fmaf(zz, fmaf(zz, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), z);
    const float c = fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    cs = k & 1 ? s : c;
    sn = k & 1 ? c : s;
    if ((k + 1) & 2) cs = -cs;
    if (k & 2) sn = -sn;
}

// RUN: heads of one token that a group of lanes takes, their loads in flight together
template <typename T, int D, bool HALF, int RUN>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    constexpr int kVec = Elem<T>::kVec;
    constexpr int kLanes = D / (2 * kVec);  // lanes of a row
    const int lane = threadIdx.x & (kLanes - 1);
    const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / kLanes;
    if (row >= a.rows) return;
    int run = blockIdx.y, which = 0;
    if (run >= a.runs[0]) {
        run -= a.runs[0];
        which = 1;
        if (run >= a.runs[1]) {
            run -= a.runs[1];
            which = 2;
        }
    }
    const air_rope_tensor &t = a.t[which];
    const int h0 = run * RUN, n_heads = a.heads[which];
    int pos[3] = {0, 0, 0};
    if (a.positions) {
        pos[0] = a.positions[row];
        if (a.n_axes > 1) pos[1] = a.positions[(int64_t)a.rows + row];
        if (a.n_axes > 2) pos[2] = a.positions[2 * (int64_t)a.rows + row];
    }
    const int b = (int)row / a.n_tokens, tok = (int)row - b * a.n_tokens;
    // the lane's two pieces: first and second elements of its pairs (half), the two parts of a run of pairs (interleaved), and
    // behind the rotated elements whatever two pieces come next
    const int half_pieces = a.pairs / kVec;
    const bool turns = lane < half_pieces && which < 2;
    const int p0 = HALF && lane < half_pieces ? lane : 2 * lane, p1 = HALF && lane < half_pieces ? lane + half_pieces : 2 * lane + 1;
    const T *src = (const T *)t.src + b * t.src_b + tok * t.src_t;
    T *dst = (T *)t.dst + b * t.dst_b + tok * t.dst_t;
    uint4 x0[RUN], x1[RUN];
#pragma unroll
    for (int r = 0; r < RUN; ++r) {
        const T *s = src + min(h0 + r, n_heads - 1) * t.src_h;
        x0[r] = *reinterpret_cast<const uint4 *>(s + kVec * p0);
        x1[r] = *reinterpret_cast<const uint4 *>(s + kVec * p1);
    }
    if (pos[0] < 0) return;  // padding (the position was requested together with the row)
    if (which < 2) {
        float cs[kVec], sn[kVec], w0[kVec], w1[kVec];
        if (t.weight) {
            unpack(*reinterpret_cast<const uint4 *>((const T *)t.weight + kVec * p0), w0);
            unpack(*reinterpret_cast<const uint4 *>((const T *)t.weight + kVec * p1), w1);
        }
        if (turns) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const int pair = kVec * lane + i;
                const int p = pair < a.end0 ? pos[0] : (pair < a.end1 ? pos[1] : pos[2]);
                turn_by((double)p, a.freqs[pair], cs[i], sn[i]);
                cs[i] *= a.scale;
                sn[i] *= a.scale;
            }
        }
#pragma unroll
        for (int r = 0; r < RUN; ++r) {
            float y0[kVec], y1[kVec];
            unpack(x0[r], y0);
            unpack(x1[r], y1);
            if (t.weight) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kVec; ++i) sum = fmaf(y0[i], y0[i], fmaf(y1[i], y1[i], sum));
#pragma unroll
                for (int m = 1; m < kLanes; m *= 2) sum += __shfl_xor(sum, m, 64);
                const float f = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    y0[i] *= f * w0[i];
                    y1[i] *= f * w1[i];
                }
            }
            if (turns) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if (HALF) {
                        const float u = y0[i], v = y1[i];
                        y0[i] = u * cs[i] - v * sn[i];
                        y1[i] = u * sn[i] + v * cs[i];
                    } else if (i < kVec / 2) {  // pairs of the first piece, then of the second
                        const float u = y0[2 * i], v = y0[2 * i + 1];
                        y0[2 * i] = u * cs[i] - v * sn[i];
                        y0[2 * i + 1] = u * sn[i] + v * cs[i];
                    } else {
                        const int j = 2 * i - kVec;
                        const float u = y1[j], v = y1[j + 1];
                        y1[j] = u * cs[i] - v * sn[i];
                        y1[j + 1] = u * sn[i] + v * cs[i];
                    }
                }
            }
            x0[r] = pack(y0);
            x1[r] = pack(y1);
        }
    }
#pragma unroll
    for (int r = 0; r < RUN; ++r) {
        if (h0 + r >= n_heads) break;
        T *o = dst + (h0 + r) * t.dst_h;
        *reinterpret_cast<uint4 *>(o + kVec * p0) = x0[r];
        *reinterpret_cast<uint4 *>(o + kVec * p1) = x1[r];
    }
}

template <typename T, int D, bool HALF>
static hipError_t rope_launch(hipStream_t s, RopeArgs &a) {
    constexpr int kLanes = D / (2 * Elem<T>::kVec), kRun = 4;
    // runs of four heads once the launch then still has 1024 workgroups or so: fewer are bound by their latency
    const bool few = a.rows * (int64_t)kLanes * (a.heads[0] + a.heads[1] + a.heads[2]) < (int64_t)kRun * 256 * 1024;
    const int threads = few ? 64 : 256, run = few ? 1 : kRun;
    int64_t runs = 0;
    for (int i = 0; i < 3; ++i) runs += a.runs[i] = (a.heads[i] + run - 1) / run;
    const dim3 grid((unsigned)(((int64_t)a.rows * kLanes + threads - 1) / threads), (unsigned)runs);
    if (few) hipLaunchKernelGGL((rope_kernel<T, D, HALF, 1>), grid, dim3(threads), 0, s, a);
    else hipLaunchKernelGGL((rope_kernel<T, D, HALF, kRun>), grid, dim3(threads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_rope(hipStream_t s, const air_rope_config &c, const air_rope_tensor *const (&t)[3], const int32_t *positions,
                       const double *freqs) {
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    for (int i = 0; i < 3; ++i) {
        if (!t[i]) continue;
        a.t[i] = *t[i];
        a.heads[i] = i == 0 ? c.n_q_heads : c.n_kv_heads;
    }
    a.n_tokens = c.n_tokens;
    a.rows = c.batch * c.n_tokens;
    a.n_axes = c.n_axes;
    a.end0 = c.axis_pairs[0];
    a.end1 = a.end0 + (c.n_axes > 1 ? c.axis_pairs[1] : 0);
    a.pairs = a.end1 + (c.n_axes > 2 ? c.axis_pairs[2] : 0);
    a.eps = c.norm_eps;
    a.scale = c.scale;
    a.positions = positions;
    a.freqs = freqs;
    const bool half = c.layout == AIR_ROPE_HALF;
    if (c.dtype == AIR_BF16)
        return c.head_dim == 128 ? (half ? rope_launch<bf16_t, 128, true>(s, a) : rope_launch<bf16_t, 128, false>(s, a))
                                 : (half ? rope_launch<bf16_t, 64, true>(s, a) : rope_launch<bf16_t, 64, false>(s, a));
    return c.head_dim == 128 ? (half ? rope_launch<float, 128, true>(s, a) : rope_launch<float, 128, false>(s, a))
                             : (half ? rope_launch<float, 64, true>(s, a) : rope_launch<float, 64, false>(s, a));
}

}  // namespace air
