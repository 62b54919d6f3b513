// air_evict: the `keep` slots of a (sequence, head) that stay, and the rows that move to make them the first ones.
//
// One workgroup per (sequence, head) finds the keep-th largest of the slots' keys by digits of 11, 11 and 10 bits (histograms in LDS, the keys there too
// where they fit), then ranks by counts of ballots: which slots below `keep` are given up, which from `keep` on stay; the i-th of the one takes
// what the i-th of the other has.  Sources lie behind `keep` and destinations in front of it, so that rows move in any order.
// Few rows are moved by the same workgroup; where there can be many, a second launch over all of the chip moves them by a list.
#include "air_device.h"
#include "air_internal.h"

namespace air {

constexpr int kEvictWaves = 16, kEvictThreads = 64 * kEvictWaves;
constexpr int kLdsKeys = 8192, kLdsMoves = 2048, kBins = 2048;
constexpr size_t kAlone = 128 << 10;  // bytes of rows that one workgroup moves by itself

struct EvictPlane {
    uint8_t *rows;
    int64_t b, h, t;
    int32_t words, wide;  // words of 16 (wide) or 4 bytes of a row
    Div by_words;
};
struct EvictArgs {
    EvictPlane p[AIR_MAX_PLANES];
    float *weights;
    int32_t *positions;
    const int32_t *lens;
    int32_t *lens_out;
    int32_t *moves;  // [pair][1 + 2 most]: count, destinations, sources; null: one launch
    int32_t n_planes, n_heads, capacity, keep, limit, first, recent, most;
    Div by_heads;
};

// Order of the slots: protected ones, NaN, then by weight (-0 like 0)
__device__ __forceinline__ uint32_t rank_key(float w, bool safe) {
    if (safe) return 0xffffffffu;
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void move_rows(const EvictArgs &a, int b, int h, int count, const int32_t *to, const int32_t *from, int first, int step) {
    for (int i = 0; i < a.n_planes; ++i) {
        const EvictPlane &p = a.p[i];
        uint8_t *rows = p.rows + b * p.b + h * p.h;
        const int total = count * p.words;  // (at most half of 2^33 bytes, in words of 4: 2^30)
        for (int x = first; x < total; x += step) {
            const int r = p.by_words.of(x), w = x - r * p.words;
            if (p.wide) {
                *reinterpret_cast<uint4 *>(rows + to[r] * p.t + 16 * w) = *reinterpret_cast<const uint4 *>(rows + from[r] * p.t + 16 * w);
            } else {
                *reinterpret_cast<uint32_t *>(rows + to[r] * p.t + 4 * w) = *reinterpret_cast<const uint32_t *>(rows + from[r] * p.t + 4 * w);
            }
        }
    }
}

__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a) {
    __shared__ uint32_t keys[kLdsKeys];
    __shared__ int32_t bins[kBins], moves[2 * kLdsMoves];
    __shared__ int32_t wave_n[3][kEvictWaves], scan[kEvictWaves + 1], found[2], last_of[kEvictWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int pair = blockIdx.x, b = a.by_heads.of(pair), h = pair - b * a.n_heads;
    int n = a.lens[b];
    n = n < 0 ? 0 : n > a.capacity ? a.capacity : n;
    const bool over = n > a.limit;
    if (h == 0 && tid == 0) a.lens_out[b] = over ? a.keep : n;
    int32_t *list = a.moves ? a.moves + (size_t)pair * (1 + 2 * (size_t)a.most) : nullptr;
    if (!over) {
        if (list && tid == 0) list[0] = 0;
        return;
    }
    float *weights = a.weights + (size_t)pair * a.capacity;
    int32_t *positions = a.positions ? a.positions + (size_t)pair * a.capacity : nullptr;

    int32_t last = INT32_MAX;  // (no position is less than 0 in front of it)
    if (positions && a.recent > 0) {
        last = INT32_MIN;
        for (int i = tid; i < n; i += kEvictThreads) last = positions[i] > last ? positions[i] : last;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int32_t o = __shfl_xor(last, s, 64);
            last = o > last ? o : last;
        }
        if (lane == 0) last_of[wave] = last;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kEvictWaves; ++w) last = last_of[w] > last ? last_of[w] : last;
    }
    const auto fetch = [&](int i) {
        bool safe = false;
        if (positions) {
            const int32_t pos = positions[i];
            safe = pos < a.first || (int64_t)last - pos < a.recent;
        }
        return rank_key(weights[i], safe);
    };
    const bool held = n <= kLdsKeys;
    if (held)
        for (int i = tid; i < n; i += kEvictThreads) keys[i] = fetch(i);
    const auto key_of = [&](int i) { return held ? keys[i] : fetch(i); };

    // ---- the keep-th largest key, and how many equal to it stay
    uint32_t value = 0, mask = 0;
    int need = a.keep;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 0x3ffu : 0x7ffu;
        for (int i = tid; i < kBins; i += kEvictThreads) bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kEvictThreads) {
            const uint32_t k = key_of(i);
            if ((k & mask) == value) atomicAdd(&bins[k >> shift & digits], 1);
        }
        __syncthreads();
        // from the top: thread t has bins 2047 - 2 t and 2046 - 2 t
        const int c0 = bins[kBins - 1 - 2 * tid], c1 = bins[kBins - 2 - 2 * tid];
        int total;
        const int above = block_excl_scan<kEvictWaves>(c0 + c1, scan, &total);
        if (above < need && need <= above + c0 + c1) {
            const bool second = need > above + c0;
            found[0] = kBins - 1 - 2 * tid - (second ? 1 : 0);
            found[1] = need - above - (second ? c0 : 0);
        }
        __syncthreads();
        value |= (uint32_t)found[0] << shift;
        mask |= digits << shift;
        need = found[1];
    }

    // ---- ranks: a wave has a run of the slots, 64 at a time
    const int run = (n + 64 * kEvictWaves - 1) / (64 * kEvictWaves) * 64, begin = wave * run, end = begin + run < n ? begin + run : n;
    int equal = 0;
    for (int i = begin; i < end; i += 64) equal += __popcll(__ballot(i + lane < end && key_of(i + lane) == value));
    if (lane == 0) wave_n[0][wave] = equal;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += wave_n[0][w];
    const uint64_t lower = (1ull << lane) - 1;
    // calls with (slot, slots given up in front of `keep` so far, staying ones behind it so far, which of the two this one is)
    const auto each = [&](auto &&f) {
        int eq = before, holes = 0, comes = 0;
        for (int i = begin; i < end; i += 64) {
            const int s = i + lane;
            const uint32_t k = s < end ? key_of(s) : 0u;
            const bool same = s < end && k == value;
            const uint64_t same_mask = __ballot(same);
            const bool stays = s < end && (k > value || (same && eq + __popcll(same_mask & lower) < need));
            const bool hole = s < end && s < a.keep && !stays, come = stays && s >= a.keep;
            const uint64_t hole_mask = __ballot(hole), come_mask = __ballot(come);
            f(s, holes + __popcll(hole_mask & lower), comes + __popcll(come_mask & lower), hole, come);
            eq += __popcll(same_mask);
            holes += __popcll(hole_mask);
            comes += __popcll(come_mask);
        }
        if (lane == 0) {
            wave_n[1][wave] = holes;
            wave_n[2][wave] = comes;
        }
    };
    each([](int, int, int, bool, bool) {});
    __syncthreads();
    int holes0 = 0, comes0 = 0, count = 0;
    for (int w = 0; w < kEvictWaves; ++w) {
        holes0 += w < wave ? wave_n[1][w] : 0;
        comes0 += w < wave ? wave_n[2][w] : 0;
        count += wave_n[1][w];
    }
    __syncthreads();
    int32_t *to = list ? list + 1 : moves, *from = to + (list ? a.most : kLdsMoves);
    each([&](int s, int holes, int comes, bool hole, bool come) {
        if (hole) to[holes0 + holes] = s;
        if (come) from[comes0 + comes] = s;
    });
    if (list && tid == 0) list[0] = count;
    __syncthreads();  // (all keys have been read; the list is written)
    for (int i = tid; i < count; i += kEvictThreads) {
        const int t = to[i], f = from[i];
        weights[t] = weights[f];
        if (positions) positions[t] = positions[f];
    }
    if (!list) move_rows(a, b, h, count, to, from, tid, kEvictThreads);
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int pair = blockIdx.y, b = a.by_heads.of(pair), h = pair - b * a.n_heads;
    const int32_t *list = a.moves + (size_t)pair * (1 + 2 * (size_t)a.most);
    move_rows(a, b, h, list[0], list + 1, list + 1 + a.most, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// rows that can move: no more than there are slots in front of `keep`, or behind it
static int64_t most_moves(const air_evict_config &c) { return c.capacity <= c.keep ? 0 : c.capacity - c.keep < c.keep ? c.capacity - c.keep : c.keep; }
static int64_t row_bytes(const air_evict_config &c) {
    int64_t n = 0;
    for (int i = 0; i < c.n_planes; ++i) n += c.planes[i].row_bytes;
    return n;
}
size_t evict_bytes(const air_evict_config &c) {
    const int64_t most = most_moves(c);
    if (c.capacity <= c.limit || (int64_t)c.batch * c.n_heads == 0) return 0;
    if (most <= kLdsMoves && most * row_bytes(c) <= (int64_t)kAlone) return 0;
    return (size_t)c.batch * c.n_heads * (1 + 2 * (size_t)most) * sizeof(int32_t);
}

hipError_t launch_evict(hipStream_t s, const air_evict_config &c, float *weights, int32_t *positions, const int32_t *lens, int32_t *lens_out,
                        void *workspace) {
    EvictArgs a;
    a.weights = weights;
    a.positions = positions;
    a.lens = lens;
    a.lens_out = lens_out;
    a.most = (int32_t)most_moves(c);
    a.moves = evict_bytes(c) ? static_cast<int32_t *>(workspace) : nullptr;
    a.n_planes = c.n_planes;
    a.n_heads = c.n_heads;
    a.capacity = c.capacity;
    a.keep = c.keep;
    a.limit = c.limit;
    a.first = c.first;
    a.recent = c.recent;
    a.by_heads = div_by(c.n_heads);
    for (int i = 0; i < c.n_planes; ++i) {
        const air_evict_plane &p = c.planes[i];
        const bool wide = aligned(p.rows, 16) && p.b % 16 == 0 && p.h % 16 == 0 && p.t % 16 == 0 && p.row_bytes % 16 == 0;
        a.p[i] = EvictPlane{static_cast<uint8_t *>(p.rows), p.b, p.h, p.t, p.row_bytes / (wide ? 16 : 4), wide, div_by(p.row_bytes / (wide ? 16 : 4))};
    }
    const int pairs = c.batch * c.n_heads;
    evict_kernel<<<pairs, kEvictThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.moves || c.n_planes == 0) return e;
    const int64_t words = ((int64_t)a.most * row_bytes(c) / 16 + 255) / 256, wgs = (2048 + pairs - 1) / pairs;
    evict_move_kernel<<<dim3((unsigned)(words < wgs ? (words < 1 ? 1 : words) : wgs), (unsigned)pairs), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace air
