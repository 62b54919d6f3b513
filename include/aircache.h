/*
 * aircache.h - C ABI of the AirCache hot path for MI355X (gfx950).
 *
 * AirCache (arxiv 2503.23956) compresses the visual part of an LVLM's KV cache once, after
 * prefill, and decodes over the shorter cache.  This library is the data-parallel part of
 * that method (Alg.1 and the decode attention of Sec.3.1):
 *
 *   air_score          Alg.1 first loop:  elite observation window (Eq.4-5), cross-modal
 *                      attention (Eq.6-7), importance I_v (Eq.8), strength and skewness
 *                      (Eq.9-10) of every layer in a range.
 *   air_budget         Eq.11: per-layer budgets from the strength / skewness of all layers.
 *   air_select_compact Alg.1 second loop: top-k by importance, gather of K / V rows into
 *                      the compacted cache.
 *   air_decode_attn    Eq.2 append + softmax(q K'^T / sqrt(d)) V' over the compacted cache.
 *
 * Around it, for the model that makes the prompt's tensors (these calls need no context):
 *
 *   air_rope           per-head norm and position rotation of queries and keys, laid out for the calls above.
 *   air_prompt_attn    causal attention of a prompt, a piece of one or a single token over the full cache.
 *
 * Behind it, for long generation (no context either):
 *
 *   air_quant_append   rows of K and V into a cache held in 4 bits; air_quant_read: what it stands for.
 *   air_quant_attn     attention over that cache: tokens, windows and pieces; what every slot was attended to.
 *   air_evict          drops the least attended tokens of a cache (4 bits, or rows of any type) in place.
 *
 * Conventions
 *   - Every tensor pointer is DEVICE memory unless its comment says "host".  Descriptor
 *     arrays (air_layer[], air_seq[]) and getter outputs are HOST memory.
 *   - The caller owns every input tensor and the workspace; the library borrows them for
 *     the duration of the enqueued work and never allocates or frees device memory.
 *   - The four stage calls only enqueue work on `stream` (a hipStream_t passed as void*;
 *     NULL = the default stream).  They do not synchronise.  The getters synchronise.
 *   - Every call returns an air_status.  Arguments are validated before anything is
 *     launched, so an error return implies that no device memory was written.
 *     air_last_error() gives a text for the last failure on that context.
 *   - Same inputs give bitwise the same outputs (no floating-point atomics anywhere).
 *   - A context is not thread-safe: the caller serialises the calls on one context.  Contexts are
 *     independent of each other.  Calls that overlap on the device (different streams) must not
 *     touch the same layers of one context.
 *   - Token layout of a prompt: [system | visual | text] (Eq.3; the system prompt is never
 *     scored and always kept).  Query head h reads KV head h / (n_q_heads / n_kv_heads).
 *   - head_dim is 64 or 128; the innermost (head_dim) axis of every tensor is contiguous.
 */
#ifndef AIRCACHE_H
#define AIRCACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct air_ctx air_ctx; /* opaque */

typedef enum {
    AIR_OK = 0,
    AIR_ERR_INVALID_ARG = 1, /* null pointer, bad enum, bad layer range                      */
    AIR_ERR_SHAPE = 2,       /* shape outside what the kernels support or the config allows */
    AIR_ERR_WORKSPACE = 3,   /* workspace missing, misaligned or too small                   */
    AIR_ERR_STATE = 4,       /* stages called out of order, decode capacity exhausted       */
    AIR_ERR_HIP = 5          /* a HIP runtime call failed; see air_last_error               */
} air_status;

typedef enum { AIR_F32 = 0, AIR_BF16 = 1 } air_dtype;

/* How Eq.11 weighs the layers (the paper's allocation and its ablations, Tab.5). */
typedef enum {
    AIR_BUDGET_STRENGTH_SKEW = 0, /* r_l = (s't + s'k)/2 * r  (Eq.11) */
    AIR_BUDGET_UNIFORM = 1,
    AIR_BUDGET_STRENGTH = 2,
    AIR_BUDGET_SKEW = 3
} air_budget_mode;

/* Which tokens serve as the observation window (Sec.3.3; window rows of the ablation table, Tab.5). */
typedef enum {
    AIR_WINDOW_TEXT = 0,  /* candidate span inside the text span, Eq.5 picks the rows (alpha = 0: all of it) */
    AIR_WINDOW_VISUAL = 1 /* the "visual window" ablation: the span lies inside the visual span (the paper
                             takes the last visual tokens) and every token of it is a row; there is no Eq.5
                             (alpha must be 0).  Row r at visual index p_r is normalised over the visual keys
                             i <= p_r (the attention it had in prefill, restricted to the visual keys as
                             Eq.7 is); no text key takes part, so Eq.9 is 1 for every layer.             */
} air_window_kind;

#define AIR_MAX_BATCH 64   /* sequences per context                       */
#define AIR_MAX_LAYERS 256 /* layers per context                          */
#define AIR_MAX_TEXT 4096  /* text tokens per sequence (candidate span)   */

typedef struct {
    int32_t n_layers, n_q_heads, n_kv_heads, head_dim, batch;
    int32_t max_vis_len;      /* largest visual span in the batch                          */
    int32_t max_nonvis_len;   /* largest (system + text) token count in the batch          */
    int32_t max_window;       /* largest candidate span (win_len) in the batch             */
    int32_t max_decode_steps; /* tokens that air_decode_attn may append per layer          */
    int32_t dtype;            /* air_dtype of Q, K, V, the compacted cache and the output  */
    int32_t budget_mode;      /* air_budget_mode                                            */
    int32_t min_keep;         /* lower bound on kept visual tokens per layer (>= 0)        */
    double alpha;             /* relevance threshold of Eq.5, in [0,1]; the paper uses 0.9 */
    double retention;         /* r: fraction of visual tokens kept overall, in (0,1]       */
    int32_t window_kind;      /* air_window_kind; 0 = the paper's text windows              */
    int32_t device_steps;     /* 0: the host counts the tokens air_decode_attn has appended and passes the
                                 count with every launch.  1 (bf16, head_dim 128 only): the count lives in
                                 device memory and advances with every decode launch that RUNS, so that a
                                 decode step captured in a HIP graph can be replayed; see air_decode_attn */
    int32_t cache_in_place;   /* 0: the compacted cache lives in the workspace.  1 (bf16, head_dim 128 only):
                                 air_select_compact compacts every layer INSIDE the prompt's own K / V tensors
                                 (App. A names the full-size cache kept until every layer is scored as the
                                 method's memory cost; this mode at least adds no second copy to it): the
                                 workspace then holds no cache pool, the layer's K / V tensors become its cache
                                 (the caller keeps them alive and no longer reads them), and decode appends
                                 into them.  Needs token stride == head_dim (each (sequence, KV head) a
                                 contiguous run of rows) and, per head, rows for the prompt plus
                                 max_decode_steps rounded up to a multiple of 32 (head stride / head_dim)    */
    int32_t causal_text;      /* 0: Eq.7 as printed, every elite row sees every elite text key.  1: an elite row
                                 sees only the elite text keys at or before its own position (what it saw in
                                 the model's causal prefill); visual keys are never masked.  Text windows only */
} air_config;

/* One prompt.  system = [0, vis_start), visual = [vis_start, vis_start+vis_len),
 * text = [vis_start+vis_len, seq_len).  [win_start, win_start+win_len) is the candidate
 * span of Eq.5, inside the text span; its last token is the reference row of Eq.4.
 * win_len == text length and alpha = 0.9 is the paper's elite window; alpha = 0 turns
 * the span into a plain continuous observation window (Tab.5).  With AIR_WINDOW_VISUAL the
 * span lies inside the visual span instead and all of it is the window. */
typedef struct {
    int32_t seq_len, vis_start, vis_len, win_start, win_len;
} air_seq;

/* One layer's tensors (device pointers). */
typedef struct {
    const void *q_text; /* [B][H_q ][text][d]: queries of the text span; row j = text token j
                           (AIR_WINDOW_VISUAL: [B][H_q][win_len][d], row j = token win_start + j) */
    const void *k;      /* [B][H_kv][seq ][d]                                                  */
    const void *v;      /* [B][H_kv][seq ][d]                                                  */
} air_layer;

/* Element strides shared by all layers of a call (innermost axis has stride 1). */
typedef struct {
    int64_t q_b, q_h, q_t;    /* q_text: batch, head, token */
    int64_t kv_b, kv_h, kv_t; /* k and v: batch, head, token */
} air_strides;

/* Bytes of device workspace a context with this config needs (0 on invalid config).  At most the last
 * n_layers * batch * n_kv_heads * ceil(max_vis_len / 256) * 32 KB of them (and, with bf16, 1/256 of that) are a stash that saves
 * air_score a second read of the visual keys; windows without a threshold of more than 32 rows per KV head have none.  fp32
 * contexts and contexts with heads of 64 elements are also created in a workspace that ends before the stash. */
size_t air_workspace_bytes(const air_config *cfg);

/* Create a context over a caller-allocated device workspace (256-byte aligned, at least
 * air_workspace_bytes(cfg)).  Clears its bookkeeping tables on the default stream and
 * waits for that.  The context itself is a small host object freed by air_destroy. */
air_status air_create(const air_config *cfg, void *workspace, size_t workspace_bytes, air_ctx **out);
air_status air_destroy(air_ctx *ctx);

/* Launch-shape overrides for tests and tuning.  They change how the work is cut into workgroups and
 * never a result; every shape they can force is a shape the library may choose by itself.  A field left
 * at 0 (select_direct_max: at -1) leaves that choice to the library, which is the state after air_create.
 * Not part of the method: no passage of the paper stands behind this call.  Nothing in the library reads
 * the environment. */
typedef struct {
    int32_t decode_splits;     /* workgroups per (layer, sequence, KV head) of air_decode_attn: 1, 2, 4, 8 or 16 */
    int32_t decode_waves;      /* wavefronts per workgroup of air_decode_attn: 1, 2, 4 or 8                     */
    int32_t decode_tiles;      /* 16-key tiles per loop iteration of a wave: 2, 4 or 8                          */
    int32_t score_block_mb;    /* MB of K_v scored per pair of passes when a window needs two passes: 1..65536   */
    int32_t score_rows_kernel; /* 1: the elite window's row parameters by their own kernel                       */
    int32_t select_threads;    /* workgroup size of the selection kernel: 256 or 512                             */
    int32_t select_direct_max; /* largest deciding bin that is ranked directly, 0..1024 (0: always the radix
                                  passes); -1: the library's default                                            */
    int32_t gather_wgs;        /* workgroups per unit of the compaction gather: 1..64                            */
    int32_t decode_order;      /* order of the units of a decode launch over all layers: 1 by layer, 2 longest
                                  cache first (where the launch shape has that variant)                         */
    int32_t decode_halves;     /* two, four or eight workgroups per unit with their part of the columns of V' each, in decode
                                  launches whose shape has that variant: 1 never, 2 whatever the number of units (the
                                  library takes it up to 128 units per launch)                                       */
    int32_t budget_in_score;   /* 1: air_score never does the allocation of Eq.11 in the tail of its last kernel
                                  (air_budget then launches the budget kernel, as it does beyond 64 layers)       */
} air_tuning;
/* AIR_ERR_INVALID_ARG (and no change) if a field holds a value outside its list. */
air_status air_set_tuning(air_ctx *ctx, const air_tuning *tuning);

/* Forget the prompt: the context returns to its state after air_create (no layer scored,
 * no budgets, empty caches) so that the next prompt of the same shape can be compressed.
 * Host bookkeeping only; nothing is enqueued and device memory is left as it is. */
air_status air_reset(air_ctx *ctx);

/* Alg.1, first loop (Eq.4-10) for layers [l0, l1).  layers: host array of l1-l0 entries;
 * seqs: host array of cfg.batch entries, the same for every call on this context (the
 * first call fixes it).  Fills importance scores and per-layer strength / skewness. */
air_status air_score(air_ctx *ctx, void *stream, int32_t l0, int32_t l1, const air_layer *layers,
                     const air_strides *strides, const air_seq *seqs);

/* Eq.11 for every sequence.  All layers must have been scored (else AIR_ERR_STATE).  Where every layer went
 * through air_score exactly once since the reset and no budgets were set by the caller, with at most 64 layers and 16 KV
 * heads, the last kernel of air_score has done the allocation in its tail and this call launches nothing; it is
 * still the call that makes the budgets available to air_select_compact.  Call it on the stream air_score ran on
 * (or one ordered behind it). */
air_status air_budget(air_ctx *ctx, void *stream);

/* Alg.1, second loop for layers [l0, l1): top-k_l visual tokens per (sequence, KV head)
 * by importance (ties to the lower token index), then K' = [K_sys ; K_v[idx] ; K_t] and
 * V' likewise into the compacted cache inside the workspace.  Needs air_budget (or
 * air_set_budgets).  After the enqueued work has run the caller may free the prompt K/V.
 * With cfg.cache_in_place the rows are instead compacted inside layers[].k / layers[].v themselves (see
 * air_config): those tensors ARE the cache afterwards and must stay alive; AIR_ERR_SHAPE if their strides or
 * rows per head do not allow it (checked for the largest budget there can be, without waiting for the device). */
air_status air_select_compact(air_ctx *ctx, void *stream, int32_t l0, int32_t l1, const air_layer *layers,
                              const air_strides *strides);

/* One decode step for layers [l0, l1): appends k_new / v_new to each layer's compacted
 * cache (Eq.2), then out[h] = softmax(q_h K'^T / sqrt(d)) V' over the whole cache
 * including the new token.  All tensors dense: q_new, out [l1-l0][B][H_q][d];
 * k_new, v_new [l1-l0][B][H_kv][d].  At most max_decode_steps calls per layer.
 * A logit of -inf weighs nothing and an infinite element of V makes its output column infinite, except in bf16 with
 * head_dim 128, where 64 keys in a row that have no other logit, and infinities in the last 32 rows, may give NaN.
 * The call enqueues kernel launches only (no copy, no memset, no allocation, no host wait), so it
 * can be recorded into a HIP graph.  With cfg.device_steps the recorded step advances the cache by
 * itself on every replay; the host then cannot check the capacity: a step that runs with the cache
 * full appends nothing, leaves `out` as it is and raises a flag that makes air_get_lengths fail
 * with AIR_ERR_STATE.  air_select_compact starts a layer's count at zero again. */
air_status air_decode_attn(air_ctx *ctx, void *stream, int32_t l0, int32_t l1, const void *q_new,
                           const void *k_new, const void *v_new, void *out);

/* air_decode_attn for callers that must not allocate and whose workspace must not serve as scratch: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * results (bit for bit) as air_decode_attn; the one difference is where the workgroups of a unit exchange
 * their split-K partials and arrival counters: in a fixed array of 8.1 MiB inside the library's device image
 * (every GPU the library runs on holds its copy until the process ends) instead of the workspace.  The call
 * allocates nothing and calls no allocating routine.
 *   - Limit: a launch that exchanges partials may have at most 1024 (unit, split) pairs, unit = (layer,
 *     sequence, KV head) of the call; beyond that the call returns AIR_ERR_SHAPE before anything is launched
 *     (pass fewer layers per call).  Launches with one workgroup per unit exchange nothing and have no limit.
 *   - The array is shared by every context and call on one GPU and keeps the last call's contents; the call
 *     clears the counters it needs with a small kernel first.  Calls that overlap on one GPU (two streams,
 *     two contexts, two threads) race on it: serialise them. */
air_status air_decode_attn_static(air_ctx *ctx, void *stream, int32_t l0, int32_t l1, const void *q_new,
                                  const void *k_new, const void *v_new, void *out);

/* ---- in front of the compression: queries and keys of the prompt, and its attention ----
 *
 * These calls need no context.  They enqueue kernels only (no allocation, no copy, no memset, no host wait), so they can be
 * recorded into a HIP graph; descriptors are read before they return.  Tensors, workspace and stream belong to the device that
 * is current.  After an error air_last_error(NULL) gives the text of the calling thread's last failure here.  They keep
 * no state: calls on different streams or threads may overlap as long as their outputs and workspaces do not.           */

typedef enum {
    AIR_ROPE_HALF = 0,       /* pair i of a head: elements i and i + pairs  */
    AIR_ROPE_INTERLEAVED = 1 /* pair i of a head: elements 2 i and 2 i + 1  */
} air_rope_layout;

typedef struct {
    int32_t n_q_heads, n_kv_heads, head_dim, dtype; /* heads of q / of k and v; head_dim 64 or 128; air_dtype           */
    int32_t batch, n_tokens;                        /* rows: batch x n_tokens, at most 2^27 (0: nothing is done)          */
    int32_t layout;                                 /* air_rope_layout                                                     */
    int32_t n_axes;                                 /* position axes, 1..3 (3: time, row and column of image tokens)       */
    int32_t axis_pairs[3];                          /* pairs that turn with axis 0, 1, 2, in the order of the pairs; their sum is a
                                                       multiple of 8, at most head_dim / 2.  Twice that many leading elements of
                                                       a head are rotated, the others pass through (0: norms and layout only)   */
    float norm_eps;                                 /* of the norms, >= 0                                                  */
    float scale;                                    /* factor of the rotated elements (1, or what air_rope_frequencies gives) */
} air_rope_config;

/* One tensor of air_rope: element strides of batch, head and token (the head_dim axis is contiguous), multiples of 16 bytes.
 * dst == src with the same strides works in place; source and destination must not overlap in any other way, nor one
 * tensor's destination another's.  A destination whose own rows overlap, whatever the strides, is refused (AIR_ERR_SHAPE).    */
typedef struct {
    const void *src;
    void *dst;
    const void *weight; /* [head_dim] of the RMS norm, in dtype; NULL: no norm.  Not for v */
    int64_t src_b, src_h, src_t, dst_b, dst_h, dst_t;
} air_rope_tensor;

/* For every row x (one token, one head) of q and k:  y = x * weight / sqrt(mean(x^2) + norm_eps)  where a weight is given, and
 * for pair i of y, turning with axis a:  angle = positions[a] * freqs[i],
 *   (y_first, y_second) -> scale * (y_first cos - y_second sin, y_first sin + y_second cos).
 * Rows of v are copied.  Any of q, k, v may be NULL (not all): that tensor is left out.  Computed in fp32 (a norm's squares too: elements
 * below 2^60, and with norm_eps 0 their root mean square above 2^-60) with angles reduced in fp64 (to 2^-28 turns up to 2^49 turns) and rounded once.
 * positions: device [n_axes][batch][n_tokens]; a row whose position on axis 0 is negative is padding: nothing is written there,
 * whatever lies in its source.  NULL only without pairs.  freqs: device [sum of axis_pairs], radians per position.         */
air_status air_rope(void *stream, const air_rope_config *cfg, const air_rope_tensor *q, const air_rope_tensor *k,
                    const air_rope_tensor *v, const int32_t *positions, const double *freqs);

/* How the frequencies are stretched for contexts longer than the model was trained on. */
typedef enum {
    AIR_ROPE_PLAIN = 0,   /* f_i = theta^(-i / n_pairs)                                                              */
    AIR_ROPE_LINEAR = 1,  /* f_i / factor                                                                            */
    AIR_ROPE_BY_PARTS = 2 /* pairs that turn at most slow_turns times in original_len positions are divided by factor, those
                             that turn at least fast_turns times stay, linear in the number of turns between; the
                             factor of the rotated elements becomes 0.1 ln(factor) + 1  (arxiv 2309.00071, Sec.3.2-3.4) */
} air_rope_scaling;

/* Host only: freqs[n_pairs] and *scale (for air_rope_config.scale; may be NULL).  theta > 0, factor >= 1; original_len, slow_turns and
 * fast_turns (the paper: 1 and 32) are read with AIR_ROPE_BY_PARTS only: original_len >= 1, 0 <= slow_turns < fast_turns. */
air_status air_rope_frequencies(int32_t n_pairs, double theta, int32_t scaling, double factor, int32_t original_len,
                                double slow_turns, double fast_turns, double *freqs, float *scale);

typedef struct {
    int32_t n_q_heads, n_kv_heads, head_dim, dtype; /* head_dim 64 or 128; air_dtype of q, k, v and out                     */
    float scale;                                    /* of the logits, > 0, at most 2^127; 0: 1 / sqrt(head_dim)            */
    int64_t q_h, q_t, k_h, k_t, v_h, v_t, out_h, out_t; /* element strides of head and token, multiples of 16 bytes; k_t and
                                                           v_t below 2^24                                              */
} air_prompt_config;

/* One sequence: where its first query, key, value and output row lie (elements from the tensors' pointers, multiples of 16 bytes:
 * sequences packed one behind the other, rows of a padded batch or pieces of larger buffers) and how many there are.  The queries are
 * the last q_len of the kv_len positions.  Lengths may be 0; kv_len at most 2^30, all sequences' queries times n_q_heads below 2^26. */
typedef struct {
    int64_t q_off, k_off, v_off, out_off;
    int32_t q_len, kv_len;
} air_prompt_seq;

/* Bytes of device workspace the call needs (0: none, or an argument that air_prompt_attn refuses).  Calls with little work per sequence are
 * split over the keys and leave partial results there. */
size_t air_prompt_workspace_bytes(const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs);

/* For query head h and query t of a sequence:  out = sum_j p_j v_j,  p = softmax over the keys j <= t + kv_len - q_len of
 * scale * q . k_j, with the keys and values of KV head h / (n_q_heads / n_kv_heads).  What lies at keys behind a row's own position, or
 * behind kv_len, counts for nothing, whatever it holds (infinities and NaN included).  A row that sees no key (q_len > kv_len), or
 * only logits of -inf, is zero.  In any other row a value that is not finite, at a key that the row sees, makes its column not finite, however
 * little the key weighs: the infinity where the weight is above 2^-120, that or no number where it is less (0 included).  Output rows
 * outside the sequences are left as they are.  Logits, maxima, sums and products are held in fp32, the products with the values before they are divided by the sum (values below 2^120 / kv_len cannot overflow there);
 * with bf16 the probabilities are rounded to bf16 for the second product; sequences of at most 32 rows (queries x query heads per KV head: single
 * tokens, steps) lose only 2^-16 of them in calls that run in tiles of 32 rows.  seqs: host array, n_seqs in 0..AIR_MAX_BATCH.
 * workspace: 256-byte aligned, free for another call when this one's work has run; may be NULL where no bytes are needed.
 * out must not overlap an input.  Output rows that overlap, of one sequence or of two, are refused (AIR_ERR_SHAPE). */
air_status air_prompt_attn(void *stream, const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs, const void *q,
                           const void *k, const void *v, void *out, void *workspace, size_t workspace_bytes);

/* ---- behind the compression: a cache in 4 bits, attention over it, eviction by attention weight ----
 *
 * As above: no context, kernels only (recordable), tensors, workspace and stream of the current device, air_last_error(NULL).  What a
 * cache holds is counted in DEVICE memory by the caller (`lens`), so that a recorded step serves every length: the calls read it when
 * they run, never change it, and clamp it to 0..capacity.                                                                     */

/* K and V in 4 bits.  Groups of `group` elements of a row share
 *   lo   = the least element, rounded down to bf16,
 *   step = (greatest - lo) / 15, rounded up to bf16; 0 where that is below 2^-120 (all codes are 0 then)
 *   code = (x - lo) / step rounded to the nearest whole number (ties to even), in 0..15
 * (difference, division by 15 and quotient rounded to fp32 each) and stand for lo + step code: off by at most step / 2 and 2^-22 of the
 * largest magnitude.  A group with an element that is not finite, or of 2^126 and more, stands for NaN throughout.
 * Memory, per (sequence, KV head, slot): codes head_dim / 2 bytes; scales head_dim / group pairs (lo, step) of bf16.
 *   V: element c in byte c / 2, even elements in the low half.  K: elements 8 p .. 8 p + 7 (p = 4 m + n, n < 4) in the four bytes
 *   from head_dim / 8 n + 4 m, of which (low half, high half) hold the elements (0, 2), (4, 6), (1, 3), (5, 7). */
typedef struct {
    int32_t batch, n_kv_heads, capacity; /* batch x n_kv_heads at most 65535; capacity slots per (sequence, KV head), 1..2^24 */
    int32_t head_dim, group;             /* 64 or 128; 32 or 64                                                                */
    int32_t dtype;                       /* air_dtype of the rows that go in and come out, of queries and outputs              */
    void *k_codes, *v_codes;   /* [batch][n_kv_heads][capacity][head_dim / 2] bytes, 16-byte aligned                         */
    void *k_scales, *v_scales; /* [batch][n_kv_heads][capacity][head_dim / group][2] bf16, 16-byte aligned                   */
} air_quant_cache;

/* Rows [batch][n_kv_heads][n_tokens] of K and V.  Strides in elements, non-negative multiples of 16 bytes.  Row t of sequence b belongs
 * to slot lens[b] + t.  Rows t >= counts[b] (NULL: n_tokens everywhere) are padding, and so are those whose slot lies outside the
 * capacity: neither the cache nor what lies at them is touched. */
typedef struct {
    void *k, *v;
    int64_t k_b, k_h, k_t, v_b, v_h, v_t;
    int32_t n_tokens;          /* batch x n_tokens at most 2^27 (0: nothing is done)                                          */
    const int32_t *lens;       /* device [batch]: slot of row 0; NULL: 0                                                      */
    const int32_t *counts;     /* device [batch]; NULL: n_tokens                                                              */
    int32_t *positions;        /* device [batch][n_kv_heads][capacity] or NULL: the slot's position, for air_evict            */
    const int32_t *first_positions; /* device [batch], with positions: of row 0 (row t: first + t)                            */
    float *weights;            /* device [batch][n_kv_heads][capacity] or NULL: the slot's weight, which starts at 0          */
} air_quant_rows;

/* Writes rows of k and v (read, not changed) into the cache, and positions and weights of their slots where given. */
air_status air_quant_append(void *stream, const air_quant_cache *cache, const air_quant_rows *rows);

/* Writes what the slots stand for to k and v (either may be NULL), rounded once.  positions, first_positions and weights must be NULL.  Rows of
 * k and of v that overlap are refused (AIR_ERR_SHAPE). */
air_status air_quant_read(void *stream, const air_quant_cache *cache, const air_quant_rows *rows);

typedef struct {
    int32_t n_q_heads, n_tokens; /* a multiple of the KV heads, at most 16384; queries of a sequence, with padding (0: nothing is done).
                                    n_tokens x n_q_heads below 2^26, times batch below 2^31                                     */
    int32_t causal;              /* 0: every query sees all slots held; 1: query t of n sees all but the last n - 1 - t        */
    int32_t max_len;             /* most slots that a sequence will hold when the call runs (0: capacity).  More are attended to all the same: the
                                    launch's shape goes by it, and whether a call is a large one (air_quant_attn)                */
    float scale;                 /* of the logits, > 0, at most 2^127; 0: 1 / sqrt(head_dim)                                  */
    const void *q;               /* [batch][n_q_heads][n_tokens][head_dim]                                                     */
    void *out;                   /* the same, or NULL: weights only                                                            */
    int64_t q_b, q_h, q_t, out_b, out_h, out_t; /* element strides, non-negative multiples of 16 bytes                        */
    const int32_t *lens;         /* device [batch]: slots held before the call                                                */
    const int32_t *counts;       /* device [batch]: queries of a sequence; NULL: n_tokens.  Rows behind them are left as they are */
    float *weights;              /* device [batch][n_kv_heads][capacity] or NULL                                               */
} air_quant_query;

/* Bytes of device workspace the call needs (0: none, or an argument that air_quant_attn refuses). */
size_t air_quant_workspace_bytes(const air_quant_cache *cache, const air_quant_query *query);

/* With `append` (its n_tokens, lens and counts those of the query) the call first does air_quant_append: the sequence then holds
 * lens + counts slots, else lens.  For query head h (KV head h / (n_q_heads / n_kv_heads)) and query t:
 *   out = sum_j p_j v_j,  p = softmax over the slots j that it sees of scale * q . k_j
 * and, with weights, weights[b][KV head][j] += sum of p_j over the queries and the query heads of the KV head, in a fixed order.
 * A query that sees no slot gives zero.  What lies in slots that a query does not see counts for nothing, whatever it stands for; a group
 * of NaN in a slot that it sees makes its part of the output (V) or all of it (K) NaN.  fp32: products of codes are exact, everything
 * else is held in fp32.  bf16: the same logits and sums, and factors p step of 15 bits for the second product.
 * Large bf16 calls round more, so that the same rows in a cache of another capacity, or with another max_len, may come out otherwise within these bounds:
 * V and the probabilities to 11 bits, 8 where groups of a slot's V lie further than 2^24 below the same group of another slot (an element of V
 * loses besides at most 2^-15 of the greatest of its group; a probability 2^-18 of the greatest among slots 32 i .. 32 i + 31, its own one of
 * them, and at most 2^-31 of its row's greatest), and without weights what K stands for to 11 bits (with them to 22; elements of K and of queries lose
 * besides at most 2^-22 of their row's greatest).  Large: with rows = n_tokens x n_q_heads / n_kv_heads above 32, slots = batch x n_kv_heads x max_len (or
 * capacity), rows x slots at least 2.6e6 (heads of 128; of 64: 6e6); with weights, of up to 224 rows, where slots are at least 32768 too, of more always.
 * Outputs are rounded once.  The sums of an output hold p up to 2^8 times the probability of the row's greatest logit, undivided: V of 2^95 and more can
 * overflow them.
 * Causal queries belong to the last counts slots of the sequence: after air_evict slots have no order, so a call of
 * more than one causal query appends its own rows.  Where lens + counts exceed the capacity, rows that have no slot are dropped, but the border still
 * counts back from the last slot: query t of n sees the first capacity - (n - 1 - t), which may lack its own.  workspace: 256-byte aligned, free for another call when this one's work has run.
 * out must not overlap an input; output rows that overlap are refused (AIR_ERR_SHAPE). */
air_status air_quant_attn(void *stream, const air_quant_cache *cache, const air_quant_query *query, const air_quant_rows *append,
                          void *workspace, size_t workspace_bytes);

#define AIR_MAX_PLANES 8
/* Rows that belong to slots: [batch][n_heads][capacity] rows of row_bytes bytes (a multiple of 4, at most 1024, 4-byte aligned; strides
 * in bytes, non-negative multiples of 4; capacity x row_bytes at most 2^33).  Rows of all planes must not overlap. */
typedef struct {
    void *rows;
    int64_t b, h, t;
    int32_t row_bytes;
} air_evict_plane;

typedef struct {
    int32_t batch, n_heads, capacity; /* batch x n_heads at most 65535; capacity 1..2^24                                  */
    int32_t keep, limit;              /* sequences with more than `limit` slots keep `keep`; 1 <= keep <= limit                */
    int32_t first, recent;            /* tokens that stay whatever they weigh; >= 0, together at most keep                     */
    int32_t n_planes;                 /* 0..AIR_MAX_PLANES                                                                     */
    air_evict_plane planes[AIR_MAX_PLANES];
} air_evict_config;

/* For every (sequence, head) with n = lens[b] > limit slots, which of them stay: first the tokens whose position is below `first`
 * or among the `recent` positions up to the largest one there; then those of the largest weights (NaN before every number, ties to the lower
 * slot), `keep` in all.  The i-th slot below `keep` that is given up takes what the i-th staying slot from `keep` on has: its rows of
 * all planes, its weight and its position.  Slots from `keep` on are left as they are.  lens_out[b] = keep, or lens[b] where
 * nothing is given up (memory of its own: every head reads lens).  positions: may be NULL with first =
 * recent = 0.  weights, positions: device [batch][n_heads][capacity].  workspace: 256-byte aligned, air_evict_workspace_bytes (0: none). */
air_status air_evict(void *stream, const air_evict_config *cfg, float *weights, int32_t *positions, const int32_t *lens, int32_t *lens_out,
                     void *workspace, size_t workspace_bytes);
size_t air_evict_workspace_bytes(const air_evict_config *cfg);

/* ---- inspection (tests, debugging): these synchronise the device ---- */
/* importance scores of layer l: host [B][H_kv][max_vis_len], the device buffer as it is (entries past a
 * sequence's vis_len are never written by the library: zero on a context that has seen one prompt) */
air_status air_get_scores(air_ctx *ctx, int32_t l, float *host);
/* elite window of layer l: counts host [B][H_q]; indices host [B][H_q][max_window] (absolute token positions) */
air_status air_get_elite(air_ctx *ctx, int32_t l, int32_t *counts, int32_t *indices);
/* per-layer strength and skewness: host [B][L] each */
air_status air_get_stats(air_ctx *ctx, double *s_t, double *s_k);
/* budgets k[b][l]: host [B][L] */
air_status air_get_budgets(air_ctx *ctx, int32_t *host);
/* replace the budgets (stage-isolated tests); every entry in [0, vis_len of b] */
air_status air_set_budgets(air_ctx *ctx, const int32_t *host);
/* kept visual indices of layer l: host [B][H_kv][max_vis_len], ascending, first k[b][l] valid */
air_status air_get_indices(air_ctx *ctx, int32_t l, int32_t *host);
/* Fix the kept visual indices of layer l instead of selecting them (same layout as air_get_indices;
 * the first k[b][l] entries of every row must be strictly ascending and inside [0, vis_len of b]):
 * air_select_compact then only gathers that layer.  With budgets of 1 this keeps the single token of
 * a chosen importance rank, the one-token-at-a-time study of Sec.4.3 (Fig.4); it also isolates the
 * gather for tests.  Needs budgets; computing or setting budgets again forgets the fixed indices. */
air_status air_set_indices(air_ctx *ctx, int32_t l, const int32_t *host);
/* current cache length (system + kept + text + appended) per (b, l): host [B][L] */
air_status air_get_lengths(air_ctx *ctx, int32_t *host);
/* rows [0, length) of the compacted cache of (layer l, sequence b, KV head h) in token
 * order, element type = cfg.dtype: host [max_rows][d] each; fails if length > max_rows */
air_status air_get_cache(air_ctx *ctx, int32_t l, int32_t b, int32_t h, void *k_host, void *v_host,
                         int32_t max_rows);

/* how air_prompt_attn would run a call: rows of a tile (32, 128 or 256) and splits over the keys.  Host only; refuses what air_prompt_attn
 * refuses of these arguments */
air_status air_prompt_plan(const air_prompt_config *cfg, const air_prompt_seq *seqs, int32_t n_seqs, int32_t *tile_rows, int32_t *splits);

/* text of the last failure on ctx; NULL: of the calling thread's last failure in a call that needs no context */
const char *air_last_error(const air_ctx *ctx);
const char *air_version(void);

#ifdef __cplusplus
}
#endif
#endif /* AIRCACHE_H */
