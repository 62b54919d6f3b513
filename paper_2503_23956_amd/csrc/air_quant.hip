// air_quant_append and air_quant_read: rows of K and V into 4 bits, and what they stand for.
//
// Bound by memory: a lane holds eight elements of a row (a group of 32 is four lanes, of 64 eight), reads them with one 16-byte access (bf16) and
// writes its eight codes as one dword; least and greatest element of a group are exchanged with DPP moves, the first lane of the group
// writes (lo, step).  Two prompts of 16 k tokens, 8 heads of 128: append 38 us (4.6 TB/s; rounding by the magic sum, reciprocals mended once in place of
// divisions: 46 before), read 28.5 (6 TB/s, the codes out of the memory-side cache); of one token of 16 sequences 3.4 and 3.0, the launch.
#include "air_device.h"
#include "air_internal.h"
#include "air_quant_dev.h"

namespace air {

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

QuantAppendArgs quant_row_args(const air_quant_cache &c, const air_quant_rows &r) {
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
    return a;
}

hipError_t launch_quant_rows(hipStream_t s, const air_quant_cache &c, const air_quant_rows &r, bool append) {
    const QuantAppendArgs a = quant_row_args(c, r);
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
