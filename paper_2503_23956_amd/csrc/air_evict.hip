// air_evict: the `keep` slots of a (sequence, head) that stay, and the rows that move to make them the first ones.
//
// One workgroup per (sequence, head) finds the keep-th largest of the slots' keys by digits of 11, 11 and 10 bits (histograms in LDS); as soon as the
// deciding digit has few slots they are ranked directly, each by comparing it with all of them.  Then counts of ballots rank which slots
// below `keep` are given up and which from `keep` on stay; the i-th of the one takes what the i-th of the other has.  Sources lie behind `keep` and
// destinations in front of it, so that rows move in any order.  Few rows are moved by the same workgroup; where there can be many, a
// second launch over all of the chip moves them by a list.
//
// A wave has a run of the slots, a lane four of them at a time; keys stay in LDS (capacities up to 24576; beyond, they are formed
// again, out of the L2 cache, wherever they are used).  What a call takes is dependent accesses, barriers and the instructions of
// one pass over code that is new to the CU: loops are not unrolled (keys in registers, 16 to 32 slots unrolled: 18 us in place of 15 at the time, one sequence of
// 7432 slots cut to 743, now 13).  16 x 4 heads of 2368 slots of which 64 go, K and V rows of 256 bytes with them: 10 us.  2 x 8 heads of 16 k slots cut
// to 8192: 21 us, and 9 for the rows.
#include "air_device.h"
#include "air_internal.h"

namespace air {

constexpr int kEvictWaves = 16, kEvictThreads = 64 * kEvictWaves;
constexpr int kCopies = 4;  // of every bin: additions of one wave to one bin take turns (16910 equal weights 8 us a pass with one copy)
constexpr int kLdsMoves = 2048, kBins = 2048, kDirect = 256;  // kDirect: slots of the deciding digit that are ranked directly
constexpr size_t kAlone = 128 << 10;  // bytes of rows that one workgroup moves by itself

struct EvictPlane {
    uint8_t *rows;
    int64_t b, h, t;
    int32_t start, wide;  // words of 16 (wide) or 4 bytes of a row lie behind those of the planes in front
};
struct EvictArgs {
    EvictPlane p[AIR_MAX_PLANES];
    float *weights;
    int32_t *positions;
    const int32_t *lens;
    int32_t *lens_out;
    int32_t *moves;  // [pair][1 + 2 most]: count, destinations, sources; null: one launch
    int32_t n_planes, n_heads, capacity, keep, limit, first, recent, most;
    int32_t words, lanes;  // words of a slot's rows in all planes; lanes that share a slot, a power of two
    Div by_heads;
};

// Order of the slots: protected ones, NaN, then by weight (-0 like 0)
__device__ __forceinline__ uint32_t rank_key(float w, bool safe) {
    const uint32_t u = __float_as_uint(w + 0.0f), k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return safe ? 0xffffffffu : w != w ? 0xfffffffeu : k;
}

// Moves slots from[i] to to[i], `lanes` threads each
struct Word {
    uint8_t *to;  // null: none
    bool wide;
    uint4 x;
};
__device__ __forceinline__ Word request(const EvictArgs &a, int b, int h, int count, const int32_t *to, const int32_t *from, int r, int w) {
    Word v = {nullptr, false, {0, 0, 0, 0}};
    if (r >= count || w >= a.words) return v;
    int64_t t = 0, off = 0;
    uint8_t *rows = nullptr;
    for (int p = 0; p < a.n_planes; ++p)
        if (w >= a.p[p].start) {
            v.wide = a.p[p].wide != 0;
            rows = a.p[p].rows;
            off = b * a.p[p].b + h * a.p[p].h + (w - a.p[p].start) * (v.wide ? 16 : 4);
            t = a.p[p].t;
        }
    rows += off;
    v.to = rows + to[r] * t;
    const uint8_t *at = rows + from[r] * t;
    if (v.wide) v.x = *reinterpret_cast<const uint4 *>(at);
    else v.x = uint4{*reinterpret_cast<const uint32_t *>(at), 0, 0, 0};
    return v;
}
__device__ __forceinline__ void put(const Word &v) {
    if (!v.to) return;
    if (v.wide) *reinterpret_cast<uint4 *>(v.to) = v.x;
    else *reinterpret_cast<uint32_t *>(v.to) = v.x.x;
}
// (six rows a thread at a time: what one workgroup moves by itself is that many fewer round trips to memory)
__device__ __forceinline__ void move_rows(const EvictArgs &a, int b, int h, int count, const int32_t *to, const int32_t *from, int thread, int threads) {
    const int step = threads / a.lanes;
    for (int w = thread & (a.lanes - 1); w < a.words; w += a.lanes)
        for (int r = thread / a.lanes; r < count; r += 6 * step) {
            const Word v0 = request(a, b, h, count, to, from, r, w), v1 = request(a, b, h, count, to, from, r + step, w);
            const Word v2 = request(a, b, h, count, to, from, r + 2 * step, w), v3 = request(a, b, h, count, to, from, r + 3 * step, w);
            const Word v4 = request(a, b, h, count, to, from, r + 4 * step, w), v5 = request(a, b, h, count, to, from, r + 5 * step, w);
            put(v0);
            put(v1);
            put(v2);
            put(v3);
            put(v4);
            put(v5);
        }
}
__device__ __forceinline__ void move_weights(float *weights, int32_t *positions, int count, const int32_t *to, const int32_t *from, int first, int step) {
    for (int i = first; i < count; i += step) {
        const int t = to[i], f = from[i];
        weights[t] = weights[f];
        if (positions) positions[t] = positions[f];
    }
}

// KEYS: slots whose keys LDS holds; 0: none
template <int KEYS>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a) {
    __shared__ __align__(16) uint32_t keys[KEYS ? KEYS : 4];
    __shared__ __align__(16) int32_t bins[kBins * kCopies];
    __shared__ int32_t moves[2 * kLdsMoves], sums[kEvictWaves], found[3], last_of[kEvictWaves];
    __shared__ uint64_t few[kDirect];  // (key, ~slot): larger goes first
    __shared__ int32_t n_few;
    __shared__ uint64_t border_at;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pair = blockIdx.x, b = a.by_heads.of(pair), h = pair - b * a.n_heads;
    float *weights = a.weights + (size_t)pair * a.capacity;
    int32_t *positions = a.positions ? a.positions + (size_t)pair * a.capacity : nullptr;
    for (int i = tid; i < kBins; i += kEvictThreads) *reinterpret_cast<int4 *>(bins + kCopies * i) = int4{0, 0, 0, 0};
    if (tid == 0) n_few = 0;
    int n = a.lens[b];
    n = n < 0 ? 0 : n > a.capacity ? a.capacity : n;
    const bool over = n > a.limit;
    if (h == 0 && tid == 0) a.lens_out[b] = over ? a.keep : n;
    int32_t *list = a.moves ? a.moves + (size_t)pair * (1 + 2 * (size_t)a.most) : nullptr;
    if (!over) {
        if (list && tid == 0) list[0] = 0;
        return;
    }
    const int run = (n + 256 * kEvictWaves - 1) / (256 * kEvictWaves) * 256, begin = wave * run, end = min(begin + run, n);

    // ---- keys
    struct Four {
        uint32_t k[4];
    };
    // four words from slot s on, in one access where they all lie in the table
    const auto fetch = [&](const void *table, int s) {
        Four v = {{0, 0, 0, 0}};
        const uint32_t *at = static_cast<const uint32_t *>(table) + s;
        if (s + 4 <= a.capacity) __builtin_memcpy(&v, at, 16);
        else
            for (int i = 0; i < 4; ++i)
                if (s + i < a.capacity) v.k[i] = at[i];
        return v;
    };
    const bool any_recent = positions && a.recent > 0, any_first = positions != nullptr;
    int32_t recent_from = 0;
    const auto settle = [&](int32_t last) {  // of the wave's slots: the first of the most recent positions
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) last = max(last, __shfl_xor(last, d, 64));
        if (lane == 0) last_of[wave] = last;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kEvictWaves; ++w) last = max(last, last_of[w]);
        const int64_t from = (int64_t)last - a.recent + 1;
        recent_from = from < INT32_MIN ? INT32_MIN : (int32_t)from;
    };
    const auto form = [&](int s, const Four &w, const Four &pos) {  // 0 for slots that are not there
        Four v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t at = (int32_t)pos.k[i];
            const uint32_t k = rank_key(__uint_as_float(w.k[i]), (any_first && at < a.first) || (any_recent && at >= recent_from));
            v.k[i] = s + i < end ? k : 0u;
        }
        return v;
    };
    if constexpr (KEYS > 0) {
        constexpr int kTurns = KEYS / (256 * kEvictWaves);
        Four w[kTurns], pos[kTurns];  // (everything requested at once)
        int32_t last = INT32_MIN;
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int s = begin + 256 * t + 4 * lane;
            if (256 * t < run && s < end) {
                w[t] = fetch(weights, s);
                if (positions) pos[t] = fetch(positions, s);
                else pos[t] = Four{{0, 0, 0, 0}};
            }
        }
        if (any_recent) {
#pragma unroll
            for (int t = 0; t < kTurns; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (256 * t < run && begin + 256 * t + 4 * lane + i < end) last = max(last, (int32_t)pos[t].k[i]);
            settle(last);
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int s = begin + 256 * t + 4 * lane;
            if (256 * t < run && s < end) {
                const Four v = form(s, w[t], pos[t]);
                *reinterpret_cast<uint4 *>(keys + s) = uint4{v.k[0], v.k[1], v.k[2], v.k[3]};
            }
        }
    } else if (any_recent) {
        int32_t last = INT32_MIN;
        for (int s = tid; s < n; s += kEvictThreads) last = max(last, positions[s]);
        settle(last);
    }
    __syncthreads();
    // f(slot, keys of it and the next three) for the wave's slots, its lanes together (begin + 256 t + 4 lane)
    const auto each = [&](auto &&f) {
#pragma unroll 1
        for (int s0 = begin; s0 < end; s0 += 256) {
            const int s = s0 + 4 * lane;
            Four v;
            if constexpr (KEYS > 0) {
                uint4 x = {0, 0, 0, 0};
                if (s < end) x = *reinterpret_cast<const uint4 *>(keys + s);
                v = Four{{x.x, x.y, x.z, x.w}};
            } else {
                v = form(s, fetch(weights, s), positions ? fetch(positions, s) : Four{{0, 0, 0, 0}});
            }
            f(s, v);
        }
    };

    // ---- the last that stays: its key, and its slot among those of its key
    uint32_t value = 0, mask = 0;
    int need = a.keep, equal = 0;
    bool direct = false;
#pragma unroll 1
    for (int pass = 0; pass < 3 && !direct; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 0x3ffu : 0x7ffu;
        if (pass > 0) {
            for (int i = tid; i < kBins; i += kEvictThreads) *reinterpret_cast<int4 *>(bins + kCopies * i) = int4{0, 0, 0, 0};
            __syncthreads();
        }
        each([&](int s, const Four &v) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s + i < end && (v.k[i] & mask) == value) atomicAdd(&bins[(v.k[i] >> shift & digits) * kCopies + (lane & (kCopies - 1))], 1);
        });
        __syncthreads();
        // from the top: thread t has bins 2047 - 2 t and 2046 - 2 t
        const int4 x0 = *reinterpret_cast<const int4 *>(bins + kCopies * (kBins - 1 - 2 * tid)), x1 = *reinterpret_cast<const int4 *>(bins + kCopies * (kBins - 2 - 2 * tid));
        const int c0 = (x0.x + x0.y) + (x0.z + x0.w), c1 = (x1.x + x1.y) + (x1.z + x1.w), mine = wave_incl_scan(c0 + c1);
        if (lane == 63) sums[wave] = mine;
        __syncthreads();
        int above = mine - c0 - c1;
#pragma unroll
        for (int w = 0; w < kEvictWaves; ++w) above += w < wave ? sums[w] : 0;
        if (above < need && need <= above + c0 + c1) {
            const bool second = need > above + c0;
            found[0] = kBins - 1 - 2 * tid - (second ? 1 : 0);
            found[1] = need - above - (second ? c0 : 0);
            found[2] = second ? c1 : c0;
        }
        __syncthreads();
        value |= (uint32_t)found[0] << shift;
        mask |= digits << shift;
        need = found[1];
        equal = found[2];
        direct = equal <= kDirect;
    }
    const auto order = [](int s, uint32_t k) { return (uint64_t)k << 32 | (uint32_t)~s; };
    if (direct) {
        each([&](int s, const Four &v) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s + i < end && (v.k[i] & mask) == value) few[atomicAdd(&n_few, 1)] = order(s + i, v.k[i]);
        });
        __syncthreads();
        // four threads share a slot's comparisons
        static_assert(4 * kDirect == kEvictThreads, "four threads a slot");
        if (64 * wave < 4 * equal) {
            const uint64_t own = tid >> 2 < equal ? few[tid >> 2] : ~0ull;
            int ahead = 0;
#pragma unroll 4
            for (int i = tid & 3; i < equal; i += 4) ahead += few[i] > own;
            ahead += __shfl_xor(ahead, 1, 64);
            ahead += __shfl_xor(ahead, 2, 64);
            if (tid >> 2 < equal && (tid & 3) == 0 && ahead == need - 1) border_at = own;
        }
    } else {  // more slots of one key: the first `need` of them stay
        int same = 0;
        const auto count_of = [&](int s, const Four &v) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) c += s + i < end && v.k[i] == value;
            return c;
        };
        each([&](int s, const Four &v) { same += count_of(s, v); });
        same = wave_incl_scan(same);
        if (lane == 63) sums[wave] = same;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < wave; ++w) before += sums[w];
        if (before < need && need <= before + sums[wave])
            each([&](int s, const Four &v) {
                const int c = count_of(s, v), upto = before + wave_incl_scan(c);
                int at = upto - c;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s + i < end && v.k[i] == value && ++at == need) border_at = order(s + i, value);
                before = __builtin_amdgcn_readlane(upto, 63);
            });
    }
    __syncthreads();
    const uint64_t border = border_at;

    // ---- slots given up in front of `keep`, staying ones from there on; counts of both in one word
    const auto which = [&](int s, const Four &v, uint32_t &holes, uint32_t &comes) {
        holes = comes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = order(s + i, v.k[i]) >= border;
            holes |= (s + i < end && s + i < a.keep && !in ? 1u : 0u) << i;
            comes |= (s + i < end && s + i >= a.keep && in ? 1u : 0u) << i;
        }
        return make_int2(__popc(holes), __popc(comes));
    };
    int2 mine = {0, 0};
    each([&](int s, const Four &v) {
        uint32_t holes, comes;
        const int2 c = which(s, v, holes, comes);
        mine.x += c.x;
        mine.y += c.y;
    });
    mine.x = wave_incl_scan(mine.x);
    mine.y = wave_incl_scan(mine.y);
    if (lane == 63) {
        sums[wave] = mine.x;
        last_of[wave] = mine.y;
    }
    __syncthreads();
    int count = 0, hole_at = 0, come_at = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
        hole_at += w < wave ? sums[w] : 0;
        come_at += w < wave ? last_of[w] : 0;
        count += sums[w];
    }
    int32_t *to = list ? list + 1 : moves, *from = to + (list ? a.most : kLdsMoves);
    each([&](int s, const Four &v) {
        uint32_t holes, comes;
        const int2 c = which(s, v, holes, comes);
        if (!__any(holes | comes)) return;
        const int h1 = hole_at + wave_incl_scan(c.x), c1 = come_at + wave_incl_scan(c.y);
        int x = h1 - c.x, y = c1 - c.y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (holes >> i & 1) to[x++] = s + i;
            if (comes >> i & 1) from[y++] = s + i;
        }
        hole_at = __builtin_amdgcn_readlane(h1, 63);
        come_at = __builtin_amdgcn_readlane(c1, 63);
    });
    if (list) {
        if (tid == 0) list[0] = count;
        return;
    }
    __syncthreads();  // (all keys have been read; the list is written)
    move_weights(weights, positions, count, to, from, tid, kEvictThreads);
    move_rows(a, b, h, count, to, from, tid, kEvictThreads);
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int pair = blockIdx.y, b = a.by_heads.of(pair), h = pair - b * a.n_heads;
    const int32_t *list = a.moves + (size_t)pair * (1 + 2 * (size_t)a.most);
    const int thread = blockIdx.x * 256 + threadIdx.x, threads = gridDim.x * 256, count = list[0];
    const size_t at = (size_t)pair * a.capacity;
    move_weights(a.weights + at, a.positions ? a.positions + at : nullptr, count, list + 1, list + 1 + a.most, thread, threads);
    move_rows(a, b, h, count, list + 1, list + 1 + a.most, thread, threads);
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
    a.words = 0;
    for (int i = 0; i < c.n_planes; ++i) {
        const air_evict_plane &p = c.planes[i];
        const bool wide = aligned(p.rows, 16) && p.b % 16 == 0 && p.h % 16 == 0 && p.t % 16 == 0 && p.row_bytes % 16 == 0;
        a.p[i] = EvictPlane{static_cast<uint8_t *>(p.rows), p.b, p.h, p.t, a.words, wide};
        a.words += p.row_bytes / (wide ? 16 : 4);
    }
    a.lanes = 1;
    while (a.lanes < a.words && a.lanes < 64) a.lanes *= 2;
    const int pairs = c.batch * c.n_heads;
    if (c.capacity <= 4096) evict_kernel<4096><<<pairs, kEvictThreads, 0, s>>>(a);
    else if (c.capacity <= 24576) evict_kernel<24576><<<pairs, kEvictThreads, 0, s>>>(a);
    else evict_kernel<0><<<pairs, kEvictThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.moves) return e;
    const int64_t words = ((int64_t)a.most * a.lanes + 1023) / 1024, wgs = (2048 + pairs - 1) / pairs;
    evict_move_kernel<<<dim3((unsigned)(words < wgs ? (words < 1 ? 1 : words) : wgs), (unsigned)pairs), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace air
