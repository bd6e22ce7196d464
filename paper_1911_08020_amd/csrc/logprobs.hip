// Log probabilities of given tokens under logits [V x B], with each column's entropy, log sum
// and most likely alternatives, and the gradient.
//
// One pass over the logits of a column keeps the running maximum m, S = sum e^(z - m) and
// U = sum e^(z - m) (z - m), rescaled when m grows; parts of a column join the same way.  Then
// lse = m + log S, log p_t = z_t - lse, entropy = log S - U / S.
//
// The alternatives come from the same pass: it keeps the maximum of every segment (what a thread
// reads), the k-th greatest of 256 groups of maxima is a bound that k logits reach, and only the
// segments whose maximum reaches it are read again.
//
// Measured on MI355X, among other calls: 10 000 x 700 fp32 feature-major 11.9 us (2.4 TB/s, two
// launches of 8 and 3) and 16.3 with five alternatives, 131 072 x 512 bf16 token-major 27.1 us (5.0
// TB/s) and 32.1 with 20, one row of 10 000 with five 8.2; the gradients of 10 000 x 700 fp32 11.1 (5.0
// TB/s) and of 50 001 x 1023 fp16 40 (5.1 TB/s).  Bound by memory where there are rows for the
// whole card, by the chain of one workgroup's loads and sums where there are few.
#include <type_traits>

#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();
// e^(z - m) is zero long before this distance; it keeps 0 * -inf out of U.
constexpr float kFar = -1e4f;
constexpr int kMaxTop = 64;
constexpr int kColThreads = 256;        // feature-major: a workgroup per (64 tokens, part)
constexpr int kColRun = 16;             // feature-major: classes of a segment, of one thread
constexpr int kJoinThreads = 256;       // to find alternatives; without, a wave
constexpr int kPartRounds = 64;         // vectors of a thread in a part, at most, to find alternatives
constexpr int kSegLanes = kColRun;      // lanes that read a segment again

struct Stat {
    float m, s, u;                      // s = 0 and u = 0 where every logit is -inf
};

// The hardware's exponential of a rounded product: off by up to (|x| + 2) 2^-23 of the term.  x is
// 0 at the greatest term and a term's share falls as e^x, so that a log sum stays within a few
// 2^-23 (and results below the smallest normal number are 0).
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    if (m == -kInf) return {m, a.s + b.s, 0.0f};
    const float da = fmaxf(a.m - m, kFar), db = fmaxf(b.m - m, kFar);
    const float ea = exp_fast(a.m - m), eb = exp_fast(b.m - m);
    return {m, a.s * ea + b.s * eb, ea * (a.u + a.s * da) + eb * (b.u + b.s * db)};
}

// The Stat of a wave's first LANES lanes, the same bits in every lane (a lane's own sum may be
// off in the last: its first addition can fuse with a product).
template <int LANES> __device__ __forceinline__ Stat join_lanes(Stat a) {
    auto over = [](float x, auto op) {
        return lane_of(group_reduce<LANES, decltype(op)>(x), LANES - 1);
    };
    const float m = over(a.m, MaxOp{});
    if (m == -kInf) return {m, over(a.s, AddOp{}), 0.0f};
    const float e = exp_fast(a.m - m), d = fmaxf(a.m - m, kFar);
    return {m, over(a.s * e, AddOp{}), over(e * (a.u + a.s * d), AddOp{})};
}

// The same sums while values come in.  The greatest value's term is 1 exactly, so that a sum is
// never below it and a log probability never above 0.
struct Sums {
    float m = -kInf, s = 0.0f, u = 0.0f;

    // to: the greater of m and the new values' maximum
    __device__ __forceinline__ void raise(float to) {
        if (to == m) return;
        const float d = fmaxf(m - to, kFar), e = exp_fast(m - to);
        u = e * (u + s * d);
        s *= e;
        m = to;
    }
    // values not above m (which is not -inf), -inf among them; a NaN or +inf makes s NaN
    template <int N> __device__ __forceinline__ void add(const float (&z)[N]) {
        float d[N], low = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            d[i] = z[i] - m;
            low = fminf(low, d[i]);
        }
        if (__any(low < kFar)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float e = exp_fast(d[i]);
                s += e;
                u = fmaf(e, fmaxf(d[i], kFar), u);
            }
        } else {                                     // nothing to keep out of U
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float e = exp_fast(d[i]);
                s += e;
                u = fmaf(e, d[i], u);
            }
        }
    }
    __device__ __forceinline__ Stat stat() const { return {m, s, u}; }
};

// The lane's V consecutive logits of a row from v on, those before `end`.  A vector that would
// pass it starts V before it instead (a row holds V at least) and leaves out its first `skip`.
template <typename T, int V> struct Run {
    Loaded<T, V> x;
    int skip;
    __device__ __forceinline__ void load(const T *row, int64_t v, int64_t end) {
        const int64_t own = v + V <= end ? v : end - V;
        skip = v - own < V ? int(v - own) : V;
        x = load_vec<T, V>(row + own);
    }
};

struct Args {
    const void *z;
    int64_t class_stride, token_stride, V, B;
    const int64_t *targets;
    int64_t top;
    float *logprob, *entropy, *lse, *top_logprob;
    int64_t *top_index;
    float4 *parts;                      // [B][nparts] Stat of each part
    uint32_t *maxima;                   // [B][nseg] orders, kept if top > 0
    int64_t nparts, nseg, part_len;
    // Token-major: the threads of a part, the vectors that each reads, the threads that share a
    // segment.  (Feature-major segments are kColRun classes.)
    int part_threads, rounds, seg_threads;
    int64_t first;                      // the launch's first row or tile
};

// ---- the k greatest -------------------------------------------------------------------

constexpr uint32_t kNanOrder = ~0u;

// A number's place in the order of logits, +0 and -0 alike.
__device__ __forceinline__ uint32_t number_order(float z) {
    const int b = __float_as_int(z + 0.0f);
    return uint32_t(b ^ (b >> 31 | int(0x80000000u)));
}
// NaN comes first.
__device__ __forceinline__ uint32_t order_of(float z) { return z != z ? kNanOrder : number_order(z); }

// The value with that order (NaN for all NaN).
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

__device__ __forceinline__ uint64_t key_at(uint64_t x, int lane) {
    return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(x >> 32), lane))) << 32 |
           uint32_t(__builtin_amdgcn_readlane(int(x), lane));
}
__device__ __forceinline__ uint64_t from_lane_below(uint64_t x) {
    constexpr int kWaveShr1 = 0x138;
    const uint32_t hi = uint32_t(x >> 32), lo = uint32_t(x);
    return uint64_t(dpp<kWaveShr1>(hi, hi)) << 32 | dpp<kWaveShr1>(lo, lo);
}

// The k greatest 64-bit keys seen so far, one per lane in descending order (0 = none).
struct TopList {
    uint64_t key = 0;
    // every lane offers a key (0 = none); all lanes take part
    __device__ __forceinline__ void offer(uint64_t mine, int k, int lane) {
        uint64_t who = __ballot(mine > key_at(key, k - 1));
        while (who) {
            const int src = __ffsll(static_cast<unsigned long long>(who)) - 1;
            const uint64_t c = key_at(mine, src);
            const int at = __popcll(__ballot(key > c));          // keys are distinct
            const uint64_t up = from_lane_below(key);
            key = lane < at ? key : lane == at ? c : up;
            who &= who - 1;
            who &= __ballot(mine > key_at(key, k - 1));
        }
    }
};

__device__ __forceinline__ uint64_t key_of(float z, uint32_t index) {
    return uint64_t(order_of(z)) << 32 | (UINT32_MAX - index);
}

// What a workgroup needs to find a token's alternatives.
constexpr int kKeys = 1024, kSegs = 1024;
struct TopRoom {
    uint64_t keys[kKeys];
    uint32_t segs[kSegs];
    uint32_t least;                     // no alternative's order is below
    uint32_t found, count;              // entries of segs, of keys
};

// f(key, rank) for those of keys[0 .. n) that have fewer than k greater ones (the keys are
// distinct): every thread counts for its own.
template <int THREADS, typename F>
__device__ __forceinline__ void ranked(const uint64_t *keys, int n, int k, F &&f) {
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t mine = keys[i];
        int rank = 0, j = 0;
        for (; j + 8 <= n; j += 8)                   // reads side by side
#pragma unroll
            for (int q = 0; q < 8; ++q) rank += keys[j + q] > mine;
        for (; j < n; ++j) rank += keys[j] > mine;
        if (rank < k) f(mine, rank);
    }
}

// The greatest x that k or more values reach, given how many reach any: by halving from lo,
// which k reach, to hi, which none passes.
template <typename F>
__device__ __forceinline__ uint32_t kth_greatest(uint32_t lo, uint32_t hi, int k, F &&reach) {
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        const int r = reach(mid);
        if (r >= k) lo = mid;
        else hi = mid - 1;
        if (r == k) break;
    }
    return lo;
}

// One wave: a bound that k or more logits reach, from n maxima of segments.  They are taken as
// 256 groups (every 256th of them): the k-th greatest of the groups' maxima is such a bound, and
// little more than k segments reach it.  Fewer than k maxima: 1, which every logit reaches.
constexpr int kGroups = 4;              // a lane
__device__ __forceinline__ uint32_t bound_of(const uint32_t *maxima, int64_t n, int k, int lane) {
    if (n < k) return 1;
    uint32_t o[kGroups] = {};
    for (int64_t i = lane; i < n; i += kGroups * kWave)
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            const int64_t at = i + q * kWave;
            const uint32_t x = at < n ? maxima[at] : 0;
            o[q] = x > o[q] ? x : o[q];
        }
    uint32_t hi = 0, lo = ~0u;                       // of the groups that have a maximum
#pragma unroll
    for (int q = 0; q < kGroups; ++q) {
        hi = o[q] > hi ? o[q] : hi;
        lo = o[q] && o[q] < lo ? o[q] : lo;
    }
    return kth_greatest(~wave_max_u32(~lo), wave_max_u32(hi), k, [&](uint32_t x) {
        int r = 0;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) r += __popcll(__ballot(o[q] >= x));
        return r;
    });
}

// The keys of a segment (-1: none) whose order is `least` at least, kSegLanes lanes together:
// f(key, or 0), with all lanes of the wave.
template <typename T, int kEach, typename F>
__device__ __forceinline__ void segment_keys(const Args &a, const T *col, int64_t seg, uint32_t least, int lane, F &&f) {
    const int in = lane % kSegLanes;
    if constexpr (kEach == 1) {
        const int64_t v = seg * kColRun + in;
        const uint64_t key = seg >= 0 && v < a.V ? key_of(float(col[v * a.class_stride]), uint32_t(v)) : 0;
        f(uint32_t(key >> 32) >= least ? key : 0);
    } else {
        // threads of a part and of a segment are powers of two
        const int seg_bits = __ffs(a.seg_threads) - 1, part_bits = __ffs(a.part_threads) - 1 - seg_bits;
        const uint32_t s = seg < 0 ? 0 : uint32_t(seg), part = s >> part_bits;
        const uint32_t thread = (s & ((1u << part_bits) - 1)) << seg_bits;
        const int64_t begin = part * a.part_len;
        int64_t end = begin + a.part_len;
        if (end > a.V) end = a.V;
        const int vectors = a.rounds * a.seg_threads;
        for (int first = 0; first < vectors; first += kSegLanes) {
            const int i = first + in, round = i >> seg_bits, t = i & (a.seg_threads - 1);
            int64_t v = begin + (int64_t(round) * a.part_threads + thread + t) * kEach;
            if (seg < 0 || i >= vectors) v = end;                    // nothing
            Run<T, kEach> x;
            x.load(col, v, end);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint64_t key = j >= x.skip ? key_of(x.x[j], uint32_t(v + j - x.skip)) : 0;
                f(uint32_t(key >> 32) >= least ? key : 0);
            }
        }
    }
}

// The alternatives of token b by a whole workgroup, given the segments' maxima (HELD: at most a
// thread's each, in LDS): the elements not below the bound, which only segments whose maximum
// reaches it hold, are collected and ranked.  Where so many are equal that there is no room for
// them, each wave goes through a share of the segments with a list of its k greatest.
template <typename T, int kEach, int THREADS, bool HELD>
__device__ __forceinline__ void write_top(const Args &a, int64_t b, const uint32_t *maxima, float lse,
                                          TopRoom &room) {
    constexpr int kWaves = THREADS / kWave, kAtOnce = kWave / kSegLanes;
    static_assert(kWaves * kMaxTop <= kKeys && THREADS % 256 == 0 && sizeof(room.keys) >= THREADS * 4, "rooms");
    const int w = wave_id(), lane = lane_id(), k = int(a.top);
    const uint32_t *groups = maxima;
    if constexpr (!HELD) {
        uint32_t most = 0;
#pragma unroll 8
        for (int64_t i = threadIdx.x; i < a.nseg; i += THREADS) most = maxima[i] > most ? maxima[i] : most;
        uint32_t *mine = reinterpret_cast<uint32_t *>(room.keys);    // not in use yet
        mine[threadIdx.x] = most;
        groups = mine;
        __syncthreads();
    }
    if (w == 0) {
        const uint32_t bound = bound_of(groups, a.nseg < THREADS ? a.nseg : THREADS, k, lane);
        if (lane == 0) {
            room.least = bound;
            room.found = room.count = 0;
        }
    }
    __syncthreads();
    const uint32_t bound = room.least;
    for (int64_t i = threadIdx.x; i < a.nseg; i += THREADS)
        if (maxima[i] >= bound) {
            const uint32_t at = atomicAdd(&room.found, 1u);
            if (at < kSegs) room.segs[at] = uint32_t(i);
        }
    __syncthreads();
    const int found = int(room.found);
    const T *col = static_cast<const T *>(a.z) + b * a.token_stride;
    if (found <= kSegs)
        for (int first = w * kAtOnce; first < found; first += kWaves * kAtOnce) {
            const int i = first + lane / kSegLanes;
            segment_keys<T, kEach>(a, col, i < found ? int64_t(room.segs[i]) : -1, bound, lane, [&](uint64_t key) {
                if (key) {
                    const uint32_t at = atomicAdd(&room.count, 1u);
                    if (at < kKeys) room.keys[at] = key;
                }
            });
        }
    __syncthreads();
    int n = int(room.count);
    if (found > kSegs || n > kKeys) {
        TopList best;
        for (int64_t first = w * kAtOnce; first < a.nseg; first += kWaves * kAtOnce) {
            const int64_t i = first + lane / kSegLanes;
            const uint32_t last = uint32_t(key_at(best.key, k - 1) >> 32), least = last > bound ? last : bound;
            const bool reaches = i < a.nseg && maxima[i] >= least;
            if (__any(reaches))
                segment_keys<T, kEach>(a, col, reaches ? i : -1, least, lane,
                                       [&](uint64_t key) { best.offer(key, k, lane); });
        }
        if (lane < k) room.keys[w * k + lane] = best.key;            // 0, which none keeps, for none
        __syncthreads();
        n = kWaves * k;
    }
    ranked<THREADS>(room.keys, n, k, [&](uint64_t key, int rank) {
        a.top_index[b * a.top + rank] = UINT32_MAX - uint32_t(key);
        a.top_logprob[b * a.top + rank] = lse == -kInf ? -kInf : value_of(uint32_t(key >> 32)) - lse;
    });
}

// A token's target and its logit, read ahead.
struct Given {
    int64_t target;
    float z;
};
template <typename T> __device__ __forceinline__ Given given_of(const Args &a, int64_t b) {
    const int64_t y = a.targets ? a.targets[b] : -1;
    const int64_t at = y < 0 || y >= a.V ? 0 : y;
    return {y, float(static_cast<const T *>(a.z)[b * a.token_stride + at * a.class_stride])};
}

// A token's results from its whole Stat, which every thread holds; its lse.
__device__ __forceinline__ float write_token(const Args &a, int64_t b, Stat t, Given y) {
    const bool empty = t.m == -kInf && t.s == 0.0f;         // nothing but -inf
    const float logs = logf(t.s), lse = empty ? -kInf : t.m + logs;
    if (threadIdx.x == 0) {
        float lp = empty ? -kInf : y.z - lse;
        if (y.target < 0) lp = 0.0f;
        if (y.target >= a.V) lp = __builtin_nanf("");
        a.logprob[b] = lp;
        a.entropy[b] = empty ? 0.0f : logs - t.u / t.s;
        a.lse[b] = lse;
    }
    return lse;
}

// ---- token-major: a row's classes are contiguous --------------------------------------

// grid (parts, B); each wave takes every kWaves-th run of 64 vectors of its part, 16
// values a lane together; the greatest value is what the wave's sums run from.  A segment is what
// a thread reads, or four neighbours where a row has several parts: no maximum crosses the wave in
// the loop, which cost a seventh of it (131 072 x 512 bf16).  A row that is one part is finished
// here, its maxima kept in LDS.
constexpr int kPartSegThreads = 4;      // of rows of several parts

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS > 256 ? 8 : 7) void rows_kernel(Args a) {
    constexpr int V = kVec<T>, kWaves = THREADS / kWave, kRun = V * kWave, kAtOnce = 16 / V;
    __shared__ Stat stats[kWaves];
    __shared__ uint32_t held[THREADS];
    __shared__ TopRoom room;
    const int w = wave_id(), lane = lane_id();
    const int64_t b = a.first + blockIdx.y, part = blockIdx.x;
    const T *row = static_cast<const T *>(a.z) + b * a.token_stride;
    const int64_t begin = part * a.part_len;
    int64_t end = begin + a.part_len;
    if (end > a.V) end = a.V;
    const Given given = a.nparts == 1 ? given_of<T>(a, b) : Given{};
    Sums t;
    float most = -kInf;                              // of the thread's elements
    bool any_nan = false;
    // the next runs are on their way while these are summed
    Loaded<T, V> x[kAtOnce];
    auto load = [&](int64_t v0) {
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int64_t v = v0 + q * (kWaves * kRun) + lane * V;
            x[q] = load_vec<T, V>(row + (v + V <= end ? v : end - V));
        }
    };
    constexpr int kRound = kAtOnce * kWaves * kRun;
    const int64_t first = begin + w * kRun;
    if (first < end) load(first);
    for (int64_t v0 = first; v0 < end; v0 += kRound) {
        float z[kAtOnce][V], m[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) z[q][i] = x[q][i];
        // a vector that would pass the end starts V before it (a row holds V at least) and leaves
        // out what others have
        if (v0 + ((kAtOnce - 1) * kWaves + 1) * kRun > end) {
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                const int64_t past = v0 + q * (kWaves * kRun) + lane * V - (end - V);
                const int skip = past > V ? V : int(past);
#pragma unroll
                for (int i = 0; i < V; ++i) z[q][i] = i >= skip ? z[q][i] : -kInf;
            }
        }
        if (v0 + kRound < end) load(v0 + kRound);
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            m[q] = z[q][0];
#pragma unroll
            for (int i = 1; i < V; ++i) m[q] = fmaxf(m[q], z[q][i]);
        }
        float all = m[0];
#pragma unroll
        for (int q = 1; q < kAtOnce; ++q) all = fmaxf(all, m[q]);
        most = fmaxf(most, all);
        if (__any(all > t.m)) t.raise(fmaxf(t.m, wave_max(all)));
        if (t.m != -kInf) {
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) t.add(z[q]);
        }
        // a NaN shows in s, or leaves no maximum: rare enough to look again
        if (__any(t.s != t.s) || t.m == -kInf) {
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                bool nan = false;
#pragma unroll
                for (int i = 0; i < V; ++i) nan |= z[q][i] != z[q][i];
                if (nan) t.s = __builtin_nanf("");
                any_nan |= nan;
            }
        }
    }
    if (a.top) {                                     // a thread without elements: that of -inf
        uint32_t order = any_nan ? kNanOrder : number_order(most);
        if (a.nparts == 1) {
            held[threadIdx.x] = order;
        } else {
            auto of = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
            order = of(order, dpp_all<kDppXor1>(order));
            order = of(order, dpp_all<kDppXor2>(order));
            if (lane % kPartSegThreads == 0)
                a.maxima[b * a.nseg + (part * THREADS + threadIdx.x) / kPartSegThreads] = order;
        }
    }
    // the wave's lanes share their maximum
    if (lane == 0) stats[w].m = t.m;
    const float sum = wave_sum(t.s), weighted = wave_sum(t.u);
    if (lane == 0) {
        stats[w].s = sum;
        stats[w].u = weighted;
    }
    __syncthreads();
    const Stat none{-kInf, 0.0f, 0.0f};
    const Stat all = join_lanes<16>(lane % 16 < kWaves ? stats[lane % 16] : none);
    if (a.nparts > 1) {
        if (threadIdx.x == 0) a.parts[b * a.nparts + part] = make_float4(all.m, all.s, all.u, 0.0f);
        return;
    }
    const float lse = write_token(a, b, all, given);
    if (a.top) write_top<T, V, THREADS, true>(a, b, held, lse, room);
}

// ---- feature-major: a class's tokens are contiguous -----------------------------------

// Workgroups go to the 8 XCDs in turn: the task of workgroup i of n such that an XCD's tasks lie
// side by side.
__device__ __forceinline__ uint32_t side_by_side(uint32_t i, uint32_t n) {
    const uint32_t xcd = i % 8, whole = n / 8, more = n % 8;
    return xcd * whole + (xcd < more ? xcd : more) + i / 8;
}

// grid (parts, token tiles of kLanes * V): a lane takes V tokens, kLanes of them a row of the
// tile; a thread takes runs of kColRun classes, each a segment.  A lane whose
// tokens would pass the end reads the last V and leaves out what the lane before it has.
template <typename T, int V, int kLanes>
__global__ __launch_bounds__(kColThreads) void columns_kernel(Args a) {
    constexpr int kRows = kColThreads / kLanes;
    __shared__ float sm[kRows][kLanes * V], ss[kRows][kLanes * V], su[kRows][kLanes * V];
    const int tx = threadIdx.x % kLanes, ty = threadIdx.x / kLanes;
    // The tiles of a part lie side by side on one XCD: they share the lines in which rows of
    // tokens are cut.
    const uint32_t task = side_by_side(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
    const int64_t part = task / gridDim.y, tile = a.first + task % gridDim.y;
    int64_t b = (tile * kLanes + tx) * V;
    int skip = 0;                                    // tokens that the lane before has
    if (b > a.B - V) {
        skip = b - (a.B - V) < V ? int(b - (a.B - V)) : V;
        b = a.B - V;
    }
    const T *z = static_cast<const T *>(a.z) + (V == 1 ? b * a.token_stride : b);
    const int64_t begin = part * a.part_len;
    int64_t end = begin + a.part_len;
    if (end > a.V) end = a.V;
    Sums t[V];
    for (int64_t v0 = begin + ty * kColRun; v0 < end; v0 += kRows * kColRun) {
        float m[V];
#pragma unroll
        for (int j = 0; j < V; ++j) m[j] = -kInf;
        // fp32: all loads of a run under way at once, which few tokens gain from (in one graph, 8
        // and 16 at once: 10 000 x 128 8.6 and 8.0 us, x 700 10.4 and 10.2, x 5000 42.8 and 41.5,
        // but 50 001 x 700 28.1 and 29.5); eight tokens of 16 bits a lane would take the registers
        // of other waves (32 000 x 2048: 35 -> 42 us)
        constexpr int kAtOnce = sizeof(T) == 4 ? kColRun : kColRun / 2;
#pragma unroll 1
        for (int r0 = 0; r0 < kColRun; r0 += kAtOnce) {
            Loaded<T, V> x[kAtOnce];
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) {
                const int64_t v = v0 + r0 + r;
                x[r] = load_vec<T, V>(z + (v < end ? v : end - 1) * a.class_stride);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float y[kAtOnce], top = m[j];
#pragma unroll
                for (int r = 0; r < kAtOnce; ++r) {
                    y[r] = v0 + r0 + r < end ? x[r][j] : -kInf;
                    top = fmaxf(top, y[r]);
                }
                t[j].raise(fmaxf(top, t[j].m));
                if (t[j].m != -kInf) t[j].add(y);
                // a NaN shows in s, or leaves no maximum: rare enough to look again
                if (t[j].s != t[j].s || top == -kInf) {
                    bool nan = m[j] != m[j];
#pragma unroll
                    for (int r = 0; r < kAtOnce; ++r) nan |= y[r] != y[r];
                    if (nan) t[j].s = top = __builtin_nanf("");
                }
                m[j] = top;
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (a.top && j >= skip) a.maxima[(b + j) * a.nseg + v0 / kColRun] = order_of(m[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const Stat mine = t[j].stat();
        sm[ty][tx * V + j] = mine.m;
        ss[ty][tx * V + j] = mine.s;
        su[ty][tx * V + j] = mine.u;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kLanes * V; i += kColThreads) {
        Stat all{sm[0][i], ss[0][i], su[0][i]};
        for (int r = 1; r < kRows; ++r) all = join(all, {sm[r][i], ss[r][i], su[r][i]});
        // where lane i / V has its tokens
        const int64_t own = (tile * kLanes + i / V) * V, at = own > a.B - V ? a.B - V : own;
        if (at + i % V >= own)
            a.parts[(at + i % V) * a.nparts + part] = make_float4(all.m, all.s, all.u, 0.0f);
    }
}

// A workgroup per token: its parts joined, the results written, the alternatives found.
template <typename T, int kEach, int THREADS>
__global__ __launch_bounds__(THREADS) void join_kernel(Args a) {
    __shared__ TopRoom room;
    const int64_t b = a.first + blockIdx.x;
    const Given given = given_of<T>(a, b);
    Stat t{-kInf, 0.0f, 0.0f};
    for (int64_t i = lane_id(); i < a.nparts; i += kWave) {       // in every wave
        const float4 p = a.parts[b * a.nparts + i];
        t = join(t, {p.x, p.y, p.z});
    }
    const float lse = write_token(a, b, join_lanes<kWave>(t), given);
    if constexpr (THREADS > kWave) write_top<T, kEach, THREADS, false>(a, b, a.maxima + b * a.nseg, lse, room);
}

// ---- the gradient ---------------------------------------------------------------------

struct GradArgs {
    const void *z;
    void *dz;
    int64_t class_stride, token_stride, out_class_stride, out_token_stride, V, B;
    const int64_t *targets;
    const float *lse, *grad_logprob, *entropy, *grad_entropy;
    int64_t first;                      // the launch's first row or tile
};

// What a token's column of the gradient needs.
struct Column {
    float lse, g, ge, h;
    int target;                                      // -1: none
};

__device__ __forceinline__ Column column_of(const GradArgs &a, float lse, int64_t target, float g, float ge, float h) {
    if (target < 0) g = 0.0f;                        // no given token
    if (target >= a.V) g = __builtin_nanf("");       // no such token
    if (lse == -kInf) lse = g = ge = h = 0.0f;       // nothing but -inf: no gradient
    return {lse, g, ge, h, target < 0 || target >= a.V ? -1 : int(target)};
}
__device__ __forceinline__ Column column_of(const GradArgs &a, int64_t b) {
    return column_of(a, a.lse[b], a.targets ? a.targets[b] : -1, a.grad_logprob ? a.grad_logprob[b] : 0.0f,
                     a.grad_entropy ? a.grad_entropy[b] : 0.0f, a.grad_entropy ? a.entropy[b] : 0.0f);
}

// p (-g - ge (log p + H)), and g more at the given token; zero where p is.
template <bool ENTROPY>
__device__ __forceinline__ float gradient(const Column &c, float z, int v) {
    const float lp = z - c.lse, p = exp_fast(lp);
    float f = -c.g;
    if (ENTROPY) f -= c.ge * (fmaxf(lp, kFar) + c.h);
    const float d = p * f;
    return v == c.target ? d + c.g : d;
}

constexpr int kGradThreads = 256;
constexpr int kColEach = 8;             // feature-major: classes of a thread

// Token-major: grid (parts of kGradThreads * 4 vectors, B).
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(kGradThreads) void grad_rows_kernel(GradArgs a) {
    constexpr int V = kVec<T>, kEach = 4;
    const int64_t b = a.first + blockIdx.y;
    const T *z = static_cast<const T *>(a.z) + b * a.token_stride;
    T *dz = static_cast<T *>(a.dz) + b * a.out_token_stride;
    const Column c = column_of(a, b);
    const int64_t base = int64_t(blockIdx.x) * (kGradThreads * kEach * V) + threadIdx.x * V;
    Loaded<T, V> x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t v = base + int64_t(i) * (kGradThreads * V);
        if (v + V <= a.V) x[i] = load_vec<T, V>(z + v);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t v = base + int64_t(i) * (kGradThreads * V);
        if (v + V <= a.V) {
            float d[V];
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = gradient<ENTROPY>(c, x[i][j], int(v + j));
            store_vec<T, V>(dz + v, d);
        } else {
            for (int64_t k = v; k < a.V; ++k) dz[k] = T(gradient<ENTROPY>(c, float(z[k]), int(k)));
        }
    }
}

// N consecutive numbers at p (none: 0).
template <int N, typename T> __device__ __forceinline__ void load_all(const T *p, int64_t at, T (&x)[N]) {
    typename VecOf<T, N>::Type v = {};
    if (p) v = *reinterpret_cast<const typename VecOf<T, N>::Type *>(p + at);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if constexpr (N == 1) x[j] = v;
        else x[j] = v[j];
    }
}

// Feature-major: threads go along the tokens, V each, and then along the classes, so that a
// workgroup reads and writes whole cache lines wherever the rows of tokens end; a thread takes
// kEach classes, a launch's `step` apart, of the same tokens.  (Tiles of 64 tokens shared lines
// with their neighbours on other XCDs: 14.6 us where this takes 11.1 for 10 000 x 700 in fp32.)  The
// last tokens of a row start where a whole vector fits; what the lane before writes too is left
// out, since dz may be z.
template <typename T, int V, bool ENTROPY>
__global__ __launch_bounds__(kGradThreads) void grad_columns_kernel(GradArgs a, uint32_t vecs, uint32_t step,
                                                                    int64_t end) {
    const uint32_t id = blockIdx.x * kGradThreads + threadIdx.x, row = id / vecs;
    if (row >= step) return;
    int64_t b = int64_t(id - row * vecs) * V;
    int skip = 0;
    if (b > a.B - V) {
        skip = int(b - (a.B - V));
        b = a.B - V;
    }
    Column c[V];
    {
        float lse[V], g[V], ge[V], h[V];
        int64_t target[V];
        load_all<V>(a.lse, b, lse);
        load_all<V>(a.targets, b, target);
        load_all<V>(a.grad_logprob, b, g);
        if (ENTROPY) {
            load_all<V>(a.grad_entropy, b, ge);
            load_all<V>(a.entropy, b, h);
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            c[j] = column_of(a, lse[j], a.targets ? target[j] : -1, g[j], ENTROPY ? ge[j] : 0.0f, ENTROPY ? h[j] : 0.0f);
    }
    const T *z = static_cast<const T *>(a.z) + b;
    T *dz = static_cast<T *>(a.dz) + b;
    const int64_t v0 = a.first + row;
    Loaded<T, V> x[kColEach];
#pragma unroll
    for (int i = 0; i < kColEach; ++i) {
        const int64_t v = v0 + int64_t(i) * step;
        x[i] = load_vec<T, V>(z + (v < end ? v : end - 1) * a.class_stride);
    }
#pragma unroll
    for (int i = 0; i < kColEach; ++i) {
        const int64_t v = v0 + int64_t(i) * step;
        if (v >= end) break;
        float d[V];
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = gradient<ENTROPY>(c[j], x[i][j], int(v));
        T *to = dz + v * a.out_class_stride;
        if (skip == 0) {
            store_vec<T, V>(to, d);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j >= skip) to[j] = T(d[j]);
        }
    }
}

// One launch per 2^15 rows or tiles of `threads` threads each, or as many as stay below 2^32 threads.
template <typename A, typename F> hipError_t over_grid_y(A a, int64_t n, int64_t threads, F &&launch) {
    constexpr int64_t kMaxGridY = 32768;
    const int64_t most = kMostThreads / threads < kMaxGridY ? kMostThreads / threads : kMaxGridY;
    for (a.first = 0; a.first < n; a.first += most) {
        launch(a, unsigned(n - a.first < most ? n - a.first : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Lanes across the tokens of a tile: the fewest vectors that hold a batch, at most 64 tokens.
int lanes_of(int64_t B, int vec) {
    int l = 1;
    while (l * vec < B && l * vec < 64) l *= 2;
    return l;
}

template <int V, typename F> hipError_t with_lanes(int lanes, F &&f) {
    if constexpr (V <= 1) if (lanes == 64) return f(std::integral_constant<int, 64>{});
    if constexpr (V <= 2) if (lanes == 32) return f(std::integral_constant<int, 32>{});
    if constexpr (V <= 4) if (lanes == 16) return f(std::integral_constant<int, 16>{});
    if (lanes == 8) return f(std::integral_constant<int, 8>{});
    if (lanes == 4) return f(std::integral_constant<int, 4>{});
    if (lanes == 2) return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1>{});
}

// How the classes of a call are cut.
struct Cut {
    bool rows;                          // token-major
    int vec, lanes;                     // feature-major
    int threads;                        // token-major
    int64_t part_len, nparts, nseg;
    int rounds, seg_threads;            // token-major
};

Cut cut_of(int dtype, int64_t V, int64_t B, bool contiguous, int64_t top) {
    Cut c;
    c.vec = dtype == DARB_F32 ? 4 : 8;
    // rows shorter than a vector go by columns, an element a lane
    c.rows = contiguous && V >= c.vec;
    if (c.rows) {
        c.lanes = 0;
        // A wave has at least four runs, or one where rows are few (one and four, fp32: 10 000 x 16
        // 4.3 and 4.5 us, x 512 6.6 and 6.4, x 1024 11.1 and 10.4; all times here in one graph).
        const int64_t run = c.vec * kWave, runs = (V + run - 1) / run, each = B < 256 ? 1 : 4;
        c.threads = 256;
        while (c.threads < 1024 && runs >= 2 * each * c.threads / kWave) c.threads *= 2;
        const int64_t step = int64_t(c.vec) * c.threads;            // one round of a workgroup
        const int64_t rounds = (V + step - 1) / step;
        // A long row several parts, two workgroups a CU in all (256, 512 and 1024 workgroups: 131 072 x
        // 64 fp32 with 5 alternatives 13.4, 12.6 and 12.6 us, without, x 256, 24.1, 26.0 and 25.5),
        // of four rounds at least: a short row's join costs more than its parts win (parts of one,
        // two and four rounds: 10 000 x 128 fp32 8.2, 4.5 and 4.5; 50 001 x 255 bf16 14.4, 14.2 and
        // 7.5; one row of 131 072 fp32 5.8, 5.8 and 5.7, with 5 alternatives 13.2, 9.9 and 8.8; one of
        // 2^20 bf16 6.2, 5.5 and 6.7, with them 29.9, 19.4 and 14.4).
        int64_t parts = (512 + B - 1) / B;
        if (parts > rounds / 4) parts = rounds / 4;
        const int64_t least = top ? (rounds + kPartRounds - 1) / kPartRounds : 1;
        if (parts < least) parts = least;
        c.rounds = int((rounds + parts - 1) / parts);
        c.part_len = c.rounds * step;
        c.nparts = (V + c.part_len - 1) / c.part_len;
        c.seg_threads = c.nparts == 1 ? 1 : kPartSegThreads;
        c.nseg = c.nparts * c.threads / c.seg_threads;
    } else {
        if (B < c.vec || contiguous) c.vec = 1;
        c.lanes = lanes_of(B, c.vec);
        const int64_t step = kColThreads / c.lanes * kColRun;     // one round of a workgroup
        const int64_t rounds = (V + step - 1) / step;
        const int64_t tiles = (B + c.lanes * c.vec - 1) / (c.lanes * c.vec);
        // four workgroups a CU (512, 1024 and 2048 in all: 10 000 x 1500 fp32 16.8, 17.5 and 17.5 us, x
        // 5000 45.7, 41.5 and 39.4, 32 000 x 2048 bf16 37.3, 34.8 and 35.3)
        int64_t parts = (1024 + tiles - 1) / tiles;
        if (parts > rounds) parts = rounds;
        c.part_len = (rounds + parts - 1) / parts * step;
        c.nparts = (V + c.part_len - 1) / c.part_len;
        c.nseg = (V + kColRun - 1) / kColRun;
        c.threads = c.rounds = c.seg_threads = 0;
    }
    return c;
}

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

int64_t logprobs_max_top() { return kMaxTop; }

// The parts of every token, and the segments' maxima; nothing where a workgroup finishes a row.
int64_t logprobs_workspace_bytes(int dtype, int64_t V, int64_t B, bool rows, int64_t top) {
    const Cut c = cut_of(dtype, V, B, rows, top);
    if (c.rows && c.nparts == 1) return 0;
    return padded(c.nparts * B * 16) + (top ? padded(c.nseg * B * 4) : 0);
}

hipError_t launch_logprobs(int dtype, int64_t V, int64_t B, bool rows, const void *z,
                           int64_t class_stride, int64_t token_stride, const int64_t *targets,
                           int64_t top, float *logprob, float *entropy, float *lse, float *top_logprob,
                           int64_t *top_index, void *workspace, hipStream_t s) {
    const Cut c = cut_of(dtype, V, B, rows, top);
    uint32_t *maxima = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + padded(c.nparts * B * 16));
    const Args a{z, class_stride, token_stride, V, B, targets, top, logprob, entropy, lse,
                 top_logprob, top_index, static_cast<float4 *>(workspace), maxima, c.nparts,
                 c.nseg, c.part_len, c.threads, c.rounds, c.seg_threads, 0};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        hipError_t e;
        if (c.rows) {
            e = over_grid_y(a, B, c.nparts * c.threads, [&](const Args &part, unsigned n) {
                const dim3 grid(unsigned(c.nparts), n);
                if (c.threads == 256)
                    hipLaunchKernelGGL((rows_kernel<T, 256>), grid, dim3(256), 0, s, part);
                else if (c.threads == 512)
                    hipLaunchKernelGGL((rows_kernel<T, 512>), grid, dim3(512), 0, s, part);
                else
                    hipLaunchKernelGGL((rows_kernel<T, 1024>), grid, dim3(1024), 0, s, part);
            });
            if (e != hipSuccess || c.nparts == 1) return e;
        } else {
            const int64_t tiles = (B + c.lanes * c.vec - 1) / (c.lanes * c.vec);
            auto columns = [&](auto vec) {
                constexpr int V1 = decltype(vec)::value;
                return with_lanes<V1>(c.lanes, [&](auto lanes) {
                    constexpr int L = decltype(lanes)::value;
                    return over_grid_y(a, tiles, c.nparts * kColThreads, [&](const Args &part, unsigned n) {
                        hipLaunchKernelGGL((columns_kernel<T, V1, L>),
                                           dim3(unsigned(c.nparts), n), dim3(kColThreads), 0, s,
                                           part);
                    });
                });
            };
            e = c.vec == 1 ? columns(std::integral_constant<int, 1>{})
                           : columns(std::integral_constant<int, kVec<T>>{});
        }
        if (e != hipSuccess) return e;
        constexpr int64_t kMost = 1 << 20;               // a launch has below 2^32 threads
        Args part = a;
        for (part.first = 0; part.first < B; part.first += kMost) {
            const dim3 grid(unsigned(B - part.first < kMost ? B - part.first : kMost));
            if (!top)
                hipLaunchKernelGGL((join_kernel<T, 1, kWave>), grid, dim3(kWave), 0, s, part);
            else if (c.rows)
                hipLaunchKernelGGL((join_kernel<T, kVec<T>, kJoinThreads>), grid, dim3(kJoinThreads), 0, s, part);
            else
                hipLaunchKernelGGL((join_kernel<T, 1, kJoinThreads>), grid, dim3(kJoinThreads), 0, s, part);
        }
        return hipGetLastError();
    });
}

hipError_t launch_logprobs_grad(int dtype, int64_t V, int64_t B, bool rows, const void *z,
                                int64_t class_stride, int64_t token_stride,
                                const int64_t *targets, const float *lse,
                                const float *grad_logprob, const float *entropy,
                                const float *grad_entropy, void *dz, int64_t out_class_stride,
                                int64_t out_token_stride, hipStream_t s) {
    const GradArgs a{z, dz, class_stride, token_stride, out_class_stride, out_token_stride, V, B,
                     targets, lse, grad_logprob, entropy, grad_entropy, 0};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        constexpr int VT = kVec<T>;
        auto launch = [&](auto with_entropy) {
            constexpr bool E = decltype(with_entropy)::value;
            if (rows) {
                const int64_t each = kGradThreads * 4 * VT, blocks = (V + each - 1) / each;
                return over_grid_y(a, B, blocks * kGradThreads, [&](const GradArgs &part, unsigned n) {
                    hipLaunchKernelGGL((grad_rows_kernel<T, E>), dim3(unsigned(blocks), n), dim3(kGradThreads), 0,
                                       s, part);
                });
            }
            const int64_t vec = B < VT ? 1 : VT, vecs = (B + vec - 1) / vec;
            GradArgs part = a;
            // a launch has below 2^32 threads
            const int64_t most = ((int64_t(1) << 31) / vecs) * kColEach;
            for (part.first = 0; part.first < V; part.first += most) {
                const int64_t end = V - part.first < most ? V : part.first + most;
                const int64_t step = (end - part.first + kColEach - 1) / kColEach;
                const dim3 grid(unsigned((step * vecs + kGradThreads - 1) / kGradThreads));
                if (vec == 1)
                    hipLaunchKernelGGL((grad_columns_kernel<T, 1, E>), grid, dim3(kGradThreads), 0, s, part,
                                       uint32_t(vecs), uint32_t(step), end);
                else
                    hipLaunchKernelGGL((grad_columns_kernel<T, VT, E>), grid, dim3(kGradThreads), 0, s, part,
                                       uint32_t(vecs), uint32_t(step), end);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        };
        return grad_entropy ? launch(std::true_type{}) : launch(std::false_type{});
    });
}

}  // namespace darb
