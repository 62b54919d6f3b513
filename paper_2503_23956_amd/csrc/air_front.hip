// Entry points that need no context (norm and rotation of queries and keys, attention over a prompt): argument checks.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "air_internal.h"

namespace air {

static thread_local char t_error[256];
const char *thread_error() { return t_error; }

static air_status refuse(air_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(t_error, sizeof(t_error), fmt, ap);
    va_end(ap);
    return st;
}

constexpr int kMaxHeads = 16384;  // runs of heads and (tile, head) pairs are grid dimensions

static bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

static const char *geometry(int hq, int hkv, int d, int dtype) {
    if (dtype != AIR_F32 && dtype != AIR_BF16) return "dtype must be AIR_F32 or AIR_BF16";
    if (d != 64 && d != 128) return "head_dim must be 64 or 128";
    if (hkv < 1 || hq < hkv || hq % hkv || hq > kMaxHeads) return "query heads must be a multiple of KV heads, at most 16384";
    return nullptr;
}

// ---- do rows that a call writes overlap?  Rows of `d` elements start at sum_i x_i stride_i; two of them overlap if their starts are less than d
// apart.  Exact, for any strides, by Euclid's algorithm: no loop over rows.
typedef __int128 wide;

static wide floor_div(wide a, wide b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// the smallest k >= 0 with low <= (a k mod m) <= high, for 0 <= low <= high < m; -1: none
static wide first_in(wide a, wide m, wide low, wide high) {
    if (low == 0) return 0;
    a %= m;
    if (a == 0) return -1;
    wide k = (low + a - 1) / a;
    if (a * k <= high) return k;
    // no multiple of a in between: the j-th turn around m has one when (m j mod a) lies between -high and -low (mod a)
    const wide j = first_in(m % a, a, (a - high % a) % a, (a - low % a) % a);
    return j < 0 ? -1 : (low + m * j + a - 1) / a;
}

struct Axis {
    int64_t stride, low, high;  // steps from low to high along it
};
// is |c + x a.stride + y b.stride| < d for some steps x, y?  An axis with steps has a stride of at least d.
static bool rows_meet(wide c, Axis a, Axis b, int64_t d) {
    if (a.low > a.high || b.low > b.high) return false;
    if (a.stride > b.stride) std::swap(a, b);
    if (b.low == b.high) {  // (then y is known; the axis with steps takes its place)
        c += (wide)b.low * b.stride;
        if (a.low == a.high) {
            c += (wide)a.low * a.stride;
            return c > -d && c < d;
        }
        std::swap(a, b);
        a = Axis{0, 0, 0};
    }
    const wide m = b.stride;
    for (int side = 0; side < 2; ++side) {  // starts 0 .. d - 1 apart, 1 .. d - 1 the other way
        const wide from = side ? 1 - d : 0, length = side ? d - 2 : d - 1;
        // w = c - from + x a.stride has to lie within `length` above a multiple -y m of m
        const wide w0 = c - from, w_low = -(wide)b.high * m, w_high = -(wide)b.low * m + m - 1;
        wide x0 = a.low, x1 = a.high;
        if (a.stride == 0) {
            if (w0 < w_low || w0 > w_high) continue;
            x1 = x0;
        } else {
            x0 = std::max(x0, -floor_div(w0 - w_low, a.stride));
            x1 = std::min(x1, floor_div(w_high - w0, a.stride));
            if (x0 > x1) continue;
        }
        const wide at = w0 + x0 * a.stride, rest = at - floor_div(at, m) * m;
        if (rest <= length) return true;
        const wide k = first_in(a.stride, m, m - rest, m - rest + length);
        if (k >= 0 && x0 + k <= x1) return true;
    }
    return false;
}

// rows of up to three axes (extent, stride): does one of them overlap another?
static bool rows_overlap(int64_t (&n)[3], int64_t (&stride)[3], int64_t d) {
    int order[3] = {0, 1, 2};
    if (n[0] == 0 || n[1] == 0 || n[2] == 0) return false;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) stride[i] = 0;
        else if (stride[i] < d) return true;
    }
    // every axis outside all that lies within its step, as tensors have it
    std::sort(order, order + 3, [&](int i, int j) { return stride[i] < stride[j]; });
    wide span = d;
    bool nested = true;
    for (int i : order) {
        if (n[i] <= 1) continue;
        nested = nested && stride[i] >= span;
        span += (wide)(n[i] - 1) * stride[i];
    }
    if (nested) return false;
    std::sort(order, order + 3, [&](int i, int j) { return n[i] < n[j]; });
    const int o = order[0], a = order[1], b = order[2];
    if (rows_meet(0, Axis{stride[a], 1, n[a] - 1}, Axis{stride[b], 1 - n[b], n[b] - 1}, d)) return true;
    for (int64_t x = 1; x < n[o]; ++x)  // (the shortest axis: at most 13003 steps in 2^27 x 2^14 rows)
        if (rows_meet((wide)x * stride[o], Axis{stride[a], 1 - n[a], n[a] - 1}, Axis{stride[b], 1 - n[b], n[b] - 1}, d)) return true;
    return false;
}

// do two sequences of a prompt attention write the same elements?
static bool sequences_overlap(const air_prompt_config &c, const air_prompt_seq *seqs, int n) {
    // what a sequence's rows span, in all and of one head, and (heads outside tokens, sequences packed along the tokens) where they start
    // inside a head's stride
    int64_t low[AIR_MAX_BATCH], span[AIR_MAX_BATCH], run[AIR_MAX_BATCH], start[AIR_MAX_BATCH], len[AIR_MAX_BATCH];
    const int64_t step = c.n_q_heads > 1 ? c.out_h : 0;
    const auto bounded = [](wide x) { return (int64_t)std::min(x, (wide)INT64_MAX); };
    int m = 0;
    for (int i = 0; i < n; ++i) {
        const air_prompt_seq &s = seqs[i];
        if (s.q_len == 0) continue;
        const wide tokens = (wide)(s.q_len - 1) * c.out_t + c.head_dim;
        low[m] = s.out_off;
        span[m] = bounded(tokens + (wide)(c.n_q_heads - 1) * c.out_h);
        run[m] = bounded(tokens);
        start[m] = step > 0 ? s.out_off % step : 0;
        len[m++] = s.q_len;
    }
    for (int i = 0; i < m; ++i)
        for (int j = 0; j < i; ++j) {
            if (low[j] - low[i] >= span[i] || low[i] - low[j] >= span[j]) continue;
            if (step > 0) {
                const int64_t x = start[j] - start[i] + (start[j] < start[i] ? step : 0);  // from i's rows on to j's, within a step
                if (x >= run[i] && run[j] <= step - x) continue;
            }
            if (rows_meet((wide)low[j] - low[i], Axis{c.out_h, 1 - c.n_q_heads, c.n_q_heads - 1}, Axis{c.out_t, 1 - len[i], len[j] - 1}, c.head_dim))
                return true;
        }
    return false;
}

}  // namespace air

using namespace air;

extern "C" {

air_status air_rope(void *stream, const air_rope_config *cfg, const air_rope_tensor *q, const air_rope_tensor *k,
                    const air_rope_tensor *v, const int32_t *positions, const double *freqs) {
    if (!cfg || (!q && !k && !v)) return refuse(AIR_ERR_INVALID_ARG, "air_rope: null argument");
    const air_rope_config &c = *cfg;
    if (const char *bad = geometry(c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype)) return refuse(AIR_ERR_SHAPE, "air_rope: %s", bad);
    if (c.batch < 0 || c.n_tokens < 0 || (int64_t)c.batch * c.n_tokens > (1 << 27))
        return refuse(AIR_ERR_SHAPE, "air_rope: batch and n_tokens must not be negative, their product at most 2^27");
    if (c.layout != AIR_ROPE_HALF && c.layout != AIR_ROPE_INTERLEAVED) return refuse(AIR_ERR_INVALID_ARG, "air_rope: unknown layout");
    if (c.n_axes < 1 || c.n_axes > 3) return refuse(AIR_ERR_INVALID_ARG, "air_rope: n_axes must be 1, 2 or 3");
    int64_t pairs = 0;
    for (int i = 0; i < c.n_axes; ++i) {
        if (c.axis_pairs[i] < 0) return refuse(AIR_ERR_SHAPE, "air_rope: negative axis_pairs");
        pairs += c.axis_pairs[i];
    }
    if (pairs % 8 || pairs > c.head_dim / 2)
        return refuse(AIR_ERR_SHAPE, "air_rope: axis_pairs must add up to a multiple of 8, at most head_dim / 2");
    if (!(c.norm_eps >= 0.f) || !isfinite(c.norm_eps) || !isfinite(c.scale))
        return refuse(AIR_ERR_INVALID_ARG, "air_rope: norm_eps must be finite and not negative, scale finite");
    const bool work = c.batch > 0 && c.n_tokens > 0;
    if (work && pairs > 0 && (!positions || !freqs)) return refuse(AIR_ERR_INVALID_ARG, "air_rope: positions and freqs are needed");
    if (!aligned(positions, 4) || !aligned(freqs, 8)) return refuse(AIR_ERR_INVALID_ARG, "air_rope: positions or freqs misaligned");
    const air_rope_tensor *const t[3] = {q, k, v};
    const int64_t vec = c.dtype == AIR_BF16 ? 8 : 4;
    for (int i = 0; i < 3; ++i) {
        if (!t[i]) continue;
        const air_rope_tensor &x = *t[i];
        const int heads = i == 0 ? c.n_q_heads : c.n_kv_heads;
        if (work && (!x.src || !x.dst)) return refuse(AIR_ERR_INVALID_ARG, "air_rope: null tensor pointer");
        if (!aligned(x.src, 16) || !aligned(x.dst, 16) || !aligned(x.weight, 16))
            return refuse(AIR_ERR_INVALID_ARG, "air_rope: tensor pointers must be 16-byte aligned");
        if (i == 2 && x.weight) return refuse(AIR_ERR_INVALID_ARG, "air_rope: values have no norm");
        const int64_t st[6] = {x.src_b, x.src_h, x.src_t, x.dst_b, x.dst_h, x.dst_t};
        for (int64_t s : st)
            if (s < 0 || s % vec) return refuse(AIR_ERR_SHAPE, "air_rope: strides must be non-negative multiples of 16 bytes");
        int64_t n[3] = {c.batch, heads, c.n_tokens}, step[3] = {x.dst_b, x.dst_h, x.dst_t};
        if (rows_overlap(n, step, c.head_dim)) return refuse(AIR_ERR_SHAPE, "air_rope: rows of a destination overlap");
        if (work && x.src == x.dst && ((c.batch > 1 && x.src_b != x.dst_b) || (heads > 1 && x.src_h != x.dst_h) || (c.n_tokens > 1 && x.src_t != x.dst_t)))
            return refuse(AIR_ERR_SHAPE, "air_rope: in place needs the same strides on both sides");
    }
    if (!work) return AIR_OK;
    const hipError_t e = launch_rope((hipStream_t)stream, c, t, positions, freqs);
    if (e != hipSuccess) return refuse(AIR_ERR_HIP, "air_rope launch: %s", hipGetErrorString(e));
    return AIR_OK;
}

air_status air_rope_frequencies(int32_t n_pairs, double theta, int32_t scaling, double factor, int32_t original_len,
                                double slow_turns, double fast_turns, double *freqs, float *scale) {
    if (n_pairs < 0 || (n_pairs > 0 && !freqs)) return refuse(AIR_ERR_INVALID_ARG, "air_rope_frequencies: null argument");
    if (scaling < AIR_ROPE_PLAIN || scaling > AIR_ROPE_BY_PARTS) return refuse(AIR_ERR_INVALID_ARG, "air_rope_frequencies: unknown scaling");
    if (!(theta > 0.0) || !isfinite(theta) || !(factor >= 1.0) || !isfinite(factor))
        return refuse(AIR_ERR_INVALID_ARG, "air_rope_frequencies: theta must be positive, factor at least 1, both finite");
    if (scaling == AIR_ROPE_BY_PARTS && (original_len < 1 || !(slow_turns >= 0.0) || !(fast_turns > slow_turns) || !isfinite(fast_turns)))
        return refuse(AIR_ERR_INVALID_ARG, "air_rope_frequencies: need original_len >= 1 and 0 <= slow_turns < fast_turns");
    constexpr double kTurn = 6.28318530717958647693;
    for (int i = 0; i < n_pairs; ++i) {
        const double f = pow(theta, -(double)i / n_pairs);
        double keep = 1.0;  // share of the frequency that is not stretched
        if (scaling == AIR_ROPE_LINEAR) keep = 0.0;
        if (scaling == AIR_ROPE_BY_PARTS) keep = fmin(1.0, fmax(0.0, (original_len * f / kTurn - slow_turns) / (fast_turns - slow_turns)));
        freqs[i] = f * keep + f / factor * (1.0 - keep);
    }
    if (scale) *scale = scaling == AIR_ROPE_BY_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return AIR_OK;
}

// what both calls of the prompt attention refuse, but for the tensors
static air_status check_prompt(const char *who, const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n, PromptPlan *plan) {
    if (!cfg || (n > 0 && !seqs)) return refuse(AIR_ERR_INVALID_ARG, "%s: null argument", who);
    const air_prompt_config &c = *cfg;
    if (const char *bad = geometry(c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype)) return refuse(AIR_ERR_SHAPE, "%s: %s", who, bad);
    if (n < 0 || n > AIR_MAX_BATCH) return refuse(AIR_ERR_SHAPE, "%s: n_seqs must be in 0..%d", who, AIR_MAX_BATCH);
    if (!(c.scale >= 0.f) || !isfinite(prompt_factor(c))) return refuse(AIR_ERR_INVALID_ARG, "%s: scale must be positive (or 0), at most 2^127", who);
    const int64_t vec = c.dtype == AIR_BF16 ? 8 : 4;
    const int64_t st[8] = {c.q_h, c.q_t, c.k_h, c.k_t, c.v_h, c.v_t, c.out_h, c.out_t};
    for (int64_t s : st)
        if (s < 0 || s % vec) return refuse(AIR_ERR_SHAPE, "%s: strides must be non-negative multiples of 16 bytes", who);
    if (c.k_t >= (1 << 24) || c.v_t >= (1 << 24)) return refuse(AIR_ERR_SHAPE, "%s: token strides of k and v must be below 2^24 elements", who);
    int32_t most = 0;
    for (int i = 0; i < n; ++i) {
        const air_prompt_seq &s = seqs[i];
        if (s.q_len < 0 || s.kv_len < 0 || s.kv_len > (1 << 30)) return refuse(AIR_ERR_SHAPE, "%s: a length is negative or above 2^30", who);
        const int64_t off[4] = {s.q_off, s.k_off, s.v_off, s.out_off};
        for (int64_t o : off)
            if (o < 0 || o % vec) return refuse(AIR_ERR_SHAPE, "%s: offsets must be non-negative multiples of 16 bytes", who);
        if (s.q_len > most) most = s.q_len;
    }
    int64_t extent[3] = {1, c.n_q_heads, most}, step[3] = {0, c.out_h, c.out_t};
    if (rows_overlap(extent, step, c.head_dim)) return refuse(AIR_ERR_SHAPE, "%s: output rows overlap", who);
    if (sequences_overlap(c, seqs, n)) return refuse(AIR_ERR_SHAPE, "%s: output rows of two sequences overlap", who);
    *plan = prompt_plan(c, seqs, n);
    if (plan->splits == 0) return refuse(AIR_ERR_SHAPE, "%s: too many rows for one call", who);
    return AIR_OK;
}

size_t air_prompt_workspace_bytes(const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs) {
    PromptPlan plan;
    return check_prompt("air_prompt_workspace_bytes", cfg, seqs, n_seqs, &plan) == AIR_OK ? plan.bytes : 0;
}

air_status air_prompt_plan(const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs, int32_t *tile_rows, int32_t *splits) {
    PromptPlan plan;
    if (!tile_rows || !splits) return refuse(AIR_ERR_INVALID_ARG, "air_prompt_plan: null argument");
    const air_status st = check_prompt("air_prompt_plan", cfg, seqs, n_seqs, &plan);
    if (st != AIR_OK) return st;
    *tile_rows = plan.tile_rows;
    *splits = plan.splits;
    return AIR_OK;
}

air_status air_prompt_attn(void *stream, const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs, const void *q,
                           const void *k, const void *v, void *out, void *workspace, size_t workspace_bytes) {
    PromptPlan plan;
    const air_status st = check_prompt("air_prompt_attn", cfg, seqs, n_seqs, &plan);
    if (st != AIR_OK) return st;
    bool rows = false, keys = false;
    for (int i = 0; i < n_seqs; ++i) {
        rows = rows || seqs[i].q_len > 0;
        keys = keys || (seqs[i].q_len > 0 && seqs[i].kv_len > 0);
    }
    if ((rows && (!q || !out)) || (keys && (!k || !v))) return refuse(AIR_ERR_INVALID_ARG, "air_prompt_attn: null tensor pointer");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
        return refuse(AIR_ERR_INVALID_ARG, "air_prompt_attn: tensors must be 16-byte aligned");
    if (plan.bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.bytes))
        return refuse(AIR_ERR_WORKSPACE, "air_prompt_attn: needs a 256-byte aligned workspace of %zu bytes", plan.bytes);
    const hipError_t e = launch_prompt((hipStream_t)stream, *cfg, plan, seqs, n_seqs, q, k, v, out, workspace);
    if (e != hipSuccess) return refuse(AIR_ERR_HIP, "air_prompt_attn launch: %s", hipGetErrorString(e));
    return AIR_OK;
}

}  // extern "C"
