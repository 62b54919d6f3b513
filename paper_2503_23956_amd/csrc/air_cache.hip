// Entry points of a cache that is generated into (4-bit rows, attention over them, eviction): argument checks.
#include <math.h>

#include <initializer_list>

#include "air_internal.h"

using namespace air;

static const char *check_cache(const air_quant_cache *c, bool pointers) {
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->group != 32 && c->group != 64) return "group must be 32 or 64";
    if (c->dtype != AIR_F32 && c->dtype != AIR_BF16) return "dtype must be AIR_F32 or AIR_BF16";
    if (c->batch < 0 || c->n_kv_heads < 1 || (int64_t)c->batch * c->n_kv_heads > 65535) return "batch x n_kv_heads must be at most 65535";
    if (c->capacity < 1 || c->capacity > (1 << 24)) return "capacity must be in 1..2^24";
    const void *const p[4] = {c->k_codes, c->v_codes, c->k_scales, c->v_scales};
    for (const void *x : p) {
        if (pointers && c->batch > 0 && !x) return "null cache pointer";
        if (!aligned(x, 16)) return "cache pointers must be 16-byte aligned";
    }
    return nullptr;
}

static bool bad_strides(int dtype, std::initializer_list<int64_t> st) {
    const int64_t vec = dtype == AIR_BF16 ? 8 : 4;
    for (int64_t s : st)
        if (s < 0 || s % vec) return true;
    return false;
}

// what append and read refuse
static air_status check_rows(const char *who, const air_quant_cache *cache, const air_quant_rows *rows, bool append, bool *work) {
    if (!cache || !rows) return refuse(AIR_ERR_INVALID_ARG, "%s: null argument", who);
    if (const char *bad = check_cache(cache, true)) return refuse(AIR_ERR_SHAPE, "%s: %s", who, bad);
    const air_quant_rows &r = *rows;
    if (r.n_tokens < 0 || (int64_t)r.n_tokens * cache->batch > (1 << 27))
        return refuse(AIR_ERR_SHAPE, "%s: n_tokens must not be negative, batch x n_tokens at most 2^27", who);
    if (!aligned(r.k, 16) || !aligned(r.v, 16)) return refuse(AIR_ERR_INVALID_ARG, "%s: k and v must be 16-byte aligned", who);
    if (!aligned(r.lens, 4) || !aligned(r.counts, 4) || !aligned(r.first_positions, 4) || !aligned(r.positions, 4) || !aligned(r.weights, 4))
        return refuse(AIR_ERR_INVALID_ARG, "%s: a table is misaligned", who);
    if (bad_strides(cache->dtype, {r.k_b, r.k_h, r.k_t, r.v_b, r.v_h, r.v_t}))
        return refuse(AIR_ERR_SHAPE, "%s: strides must be non-negative multiples of 16 bytes", who);
    *work = cache->batch > 0 && r.n_tokens > 0;
    if (append) {
        if (*work && (!r.k || !r.v)) return refuse(AIR_ERR_INVALID_ARG, "%s: null tensor pointer", who);
        if (r.positions && !r.first_positions) return refuse(AIR_ERR_INVALID_ARG, "%s: positions need first_positions", who);
    } else {
        if (r.positions || r.first_positions || r.weights) return refuse(AIR_ERR_INVALID_ARG, "%s: takes no positions and weights", who);
        if (*work && !r.k && !r.v) return refuse(AIR_ERR_INVALID_ARG, "%s: one of k and v is needed", who);
        int64_t n[3] = {cache->batch, cache->n_kv_heads, r.n_tokens}, k[3] = {r.k_b, r.k_h, r.k_t}, v[3] = {r.v_b, r.v_h, r.v_t};
        if (r.k && rows_overlap(n, k, cache->head_dim)) return refuse(AIR_ERR_SHAPE, "%s: rows of k overlap", who);
        if (r.v && rows_overlap(n, v, cache->head_dim)) return refuse(AIR_ERR_SHAPE, "%s: rows of v overlap", who);
    }
    return AIR_OK;
}

static air_status run_rows(const char *who, void *stream, const air_quant_cache *cache, const air_quant_rows *rows, bool append) {
    bool work = false;
    const air_status st = check_rows(who, cache, rows, append, &work);
    if (st != AIR_OK || !work) return st;
    const hipError_t e = launch_quant_rows((hipStream_t)stream, *cache, *rows, append);
    return e == hipSuccess ? AIR_OK : refuse(AIR_ERR_HIP, "%s launch: %s", who, hipGetErrorString(e));
}

static air_status check_query(const char *who, const air_quant_cache *cache, const air_quant_query *query, bool pointers, QuantPlan *plan) {
    if (!cache || !query) return refuse(AIR_ERR_INVALID_ARG, "%s: null argument", who);
    if (const char *bad = check_cache(cache, pointers)) return refuse(AIR_ERR_SHAPE, "%s: %s", who, bad);
    const air_quant_query &q = *query;
    if (const char *bad = geometry(q.n_q_heads, cache->n_kv_heads, cache->head_dim, cache->dtype)) return refuse(AIR_ERR_SHAPE, "%s: %s", who, bad);
    if (q.n_tokens < 0 || (int64_t)q.n_tokens * q.n_q_heads >= (1 << 26))
        return refuse(AIR_ERR_SHAPE, "%s: n_tokens must not be negative, n_tokens x n_q_heads below 2^26", who);
    if ((int64_t)q.n_tokens * q.n_q_heads * cache->batch >= (1ll << 31))
        return refuse(AIR_ERR_SHAPE, "%s: batch x n_tokens x n_q_heads must be below 2^31", who);
    if (q.causal != 0 && q.causal != 1) return refuse(AIR_ERR_INVALID_ARG, "%s: causal must be 0 or 1", who);
    if (q.max_len < 0) return refuse(AIR_ERR_INVALID_ARG, "%s: max_len must not be negative", who);
    if (!(q.scale >= 0.f) || !isfinite(logit_factor(q.scale, cache->head_dim)))
        return refuse(AIR_ERR_INVALID_ARG, "%s: scale must be positive (or 0), at most 2^127", who);
    if (bad_strides(cache->dtype, {q.q_b, q.q_h, q.q_t, q.out_b, q.out_h, q.out_t}))
        return refuse(AIR_ERR_SHAPE, "%s: strides must be non-negative multiples of 16 bytes", who);
    int64_t n[3] = {cache->batch, q.n_q_heads, q.n_tokens}, step[3] = {q.out_b, q.out_h, q.out_t};
    if (q.out && rows_overlap(n, step, cache->head_dim)) return refuse(AIR_ERR_SHAPE, "%s: output rows overlap", who);
    *plan = quant_plan(*cache, q);
    return AIR_OK;
}

static air_status check_evict(const char *who, const air_evict_config *cfg) {
    if (!cfg) return refuse(AIR_ERR_INVALID_ARG, "%s: null argument", who);
    const air_evict_config &c = *cfg;
    if (c.batch < 0 || c.n_heads < 1 || (int64_t)c.batch * c.n_heads > 65535) return refuse(AIR_ERR_SHAPE, "%s: batch x n_heads must be at most 65535", who);
    if (c.capacity < 1 || c.capacity > (1 << 24)) return refuse(AIR_ERR_SHAPE, "%s: capacity must be in 1..2^24", who);
    if (c.keep < 1 || c.limit < c.keep) return refuse(AIR_ERR_INVALID_ARG, "%s: need 1 <= keep <= limit", who);
    if (c.first < 0 || c.recent < 0 || (int64_t)c.first + c.recent > c.keep)
        return refuse(AIR_ERR_INVALID_ARG, "%s: first and recent must not be negative, together at most keep", who);
    if (c.n_planes < 0 || c.n_planes > AIR_MAX_PLANES) return refuse(AIR_ERR_INVALID_ARG, "%s: n_planes must be in 0..%d", who, AIR_MAX_PLANES);
    for (int i = 0; i < c.n_planes; ++i) {
        const air_evict_plane &p = c.planes[i];
        if (!aligned(p.rows, 4)) return refuse(AIR_ERR_INVALID_ARG, "%s: planes must be 4-byte aligned", who);
        if (p.row_bytes < 4 || p.row_bytes > 1024 || p.row_bytes % 4)
            return refuse(AIR_ERR_SHAPE, "%s: row_bytes must be a multiple of 4, at most 1024", who);
        if ((int64_t)c.capacity * p.row_bytes > (1ll << 33)) return refuse(AIR_ERR_SHAPE, "%s: capacity x row_bytes must be at most 2^33", who);
        if (p.b < 0 || p.h < 0 || p.t < 0 || p.b % 4 || p.h % 4 || p.t % 4)
            return refuse(AIR_ERR_SHAPE, "%s: strides must be non-negative multiples of 4 bytes", who);
        int64_t n[3] = {c.batch, c.n_heads, c.capacity}, step[3] = {p.b, p.h, p.t};
        if (rows_overlap(n, step, p.row_bytes)) return refuse(AIR_ERR_SHAPE, "%s: rows of a plane overlap", who);
    }
    return AIR_OK;
}

extern "C" {

air_status air_quant_append(void *stream, const air_quant_cache *cache, const air_quant_rows *rows) {
    return run_rows("air_quant_append", stream, cache, rows, true);
}

air_status air_quant_read(void *stream, const air_quant_cache *cache, const air_quant_rows *rows) {
    return run_rows("air_quant_read", stream, cache, rows, false);
}

size_t air_quant_workspace_bytes(const air_quant_cache *cache, const air_quant_query *query) {
    QuantPlan plan;
    return check_query("air_quant_workspace_bytes", cache, query, false, &plan) == AIR_OK ? plan.bytes : 0;
}

air_status air_quant_attn(void *stream, const air_quant_cache *cache, const air_quant_query *query, const air_quant_rows *append,
                          void *workspace, size_t workspace_bytes) {
    QuantPlan plan;
    air_status st = check_query("air_quant_attn", cache, query, true, &plan);
    if (st != AIR_OK) return st;
    const air_quant_query &q = *query;
    const bool work = cache->batch > 0 && q.n_tokens > 0;
    if (work && (!q.q || !q.lens || (!q.out && !q.weights))) return refuse(AIR_ERR_INVALID_ARG, "air_quant_attn: q, lens and one of out and weights are needed");
    if (!aligned(q.q, 16) || !aligned(q.out, 16)) return refuse(AIR_ERR_INVALID_ARG, "air_quant_attn: tensors must be 16-byte aligned");
    if (!aligned(q.lens, 4) || !aligned(q.counts, 4) || !aligned(q.weights, 4)) return refuse(AIR_ERR_INVALID_ARG, "air_quant_attn: a table is misaligned");
    bool rows = false;
    if (append) {
        st = check_rows("air_quant_attn", cache, append, true, &rows);
        if (st != AIR_OK) return st;
        if (append->n_tokens != q.n_tokens || append->lens != q.lens || append->counts != q.counts)
            return refuse(AIR_ERR_INVALID_ARG, "air_quant_attn: n_tokens, lens and counts of the rows must be those of the query");
    }
    if (!work) return AIR_OK;
    if (plan.bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.bytes))
        return refuse(AIR_ERR_WORKSPACE, "air_quant_attn: needs a 256-byte aligned workspace of %zu bytes", plan.bytes);
    const hipError_t e = launch_quant_attn((hipStream_t)stream, *cache, plan, q, append, workspace);
    return e == hipSuccess ? AIR_OK : refuse(AIR_ERR_HIP, "air_quant_attn launch: %s", hipGetErrorString(e));
}

size_t air_evict_workspace_bytes(const air_evict_config *cfg) {
    return check_evict("air_evict_workspace_bytes", cfg) == AIR_OK ? evict_bytes(*cfg) : 0;
}

air_status air_evict(void *stream, const air_evict_config *cfg, float *weights, int32_t *positions, const int32_t *lens, int32_t *lens_out,
                     void *workspace, size_t workspace_bytes) {
    const air_status st = check_evict("air_evict", cfg);
    if (st != AIR_OK) return st;
    const air_evict_config &c = *cfg;
    if (!aligned(weights, 4) || !aligned(positions, 4) || !aligned(lens, 4) || !aligned(lens_out, 4))
        return refuse(AIR_ERR_INVALID_ARG, "air_evict: a table is misaligned");
    if (!positions && (c.first > 0 || c.recent > 0)) return refuse(AIR_ERR_INVALID_ARG, "air_evict: first and recent need positions");
    if (c.batch == 0) return AIR_OK;
    if (!weights || !lens || !lens_out) return refuse(AIR_ERR_INVALID_ARG, "air_evict: null argument");
    if (lens < lens_out + c.batch && lens_out < lens + c.batch) return refuse(AIR_ERR_INVALID_ARG, "air_evict: lens_out must not overlap lens");
    for (int i = 0; i < c.n_planes; ++i)
        if (!c.planes[i].rows) return refuse(AIR_ERR_INVALID_ARG, "air_evict: null plane");
    const size_t bytes = evict_bytes(c);
    if (bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < bytes))
        return refuse(AIR_ERR_WORKSPACE, "air_evict: needs a 256-byte aligned workspace of %zu bytes", bytes);
    const hipError_t e = launch_evict((hipStream_t)stream, c, weights, positions, lens, lens_out, workspace);
    return e == hipSuccess ? AIR_OK : refuse(AIR_ERR_HIP, "air_evict launch: %s", hipGetErrorString(e));
}

}  // extern "C"
