// Log probabilities of given tokens under logits [V x B], with each column's entropy, log sum
// and most likely alternatives, and the gradient.
//
// One pass over the logits of a column keeps the running maximum m, S = sum e^(z - m) and
// U = sum e^(z - m) (z - m), rescaled when m grows; parts of a column join the same way.  Then
// lse = m + log S, log p_t = z_t - lse, entropy = log S - U / S.
//
// The alternatives come from the same pass: it keeps the maximum of every segment (a run of
// consecutive classes), the k greatest logits lie in the k segments with the greatest maxima
// (of equal ones the earlier segments), and only those segments are read again.
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
constexpr int kRowThreads = 256;        // token-major: a workgroup per part of a row
constexpr int kColThreads = 256;        // feature-major: a workgroup per (64 tokens, part)
constexpr int kColRun = 16;             // feature-major: classes of a segment, of one thread
constexpr int kJoinThreads = 256;

struct Stat {
    float m, s, u;                      // s = 0 and u = 0 where every logit is -inf
};

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    if (m == -kInf) return {m, a.s + b.s, 0.0f};
    const float da = fmaxf(a.m - m, kFar), db = fmaxf(b.m - m, kFar);
    const float ea = exp_fast(a.m - m), eb = exp_fast(b.m - m);
    return {m, a.s * ea + b.s * eb, ea * (a.u + a.s * da) + eb * (b.u + b.s * db)};
}

__device__ __forceinline__ Stat shuffle_xor(Stat a, int d) {
    return {__shfl_xor(a.m, d, kWave), __shfl_xor(a.s, d, kWave), __shfl_xor(a.u, d, kWave)};
}

// Adds n values to a running Stat; m is their maximum and the old maximum's (an infinite or
// NaN logit makes s NaN: z - m is, or e^(z - m) is).
template <int N> __device__ __forceinline__ void add_values(Stat &t, const float (&z)[N], float m) {
    if (m == -kInf) return;
    if (m != t.m) {
        const float d = fmaxf(t.m - m, kFar), e = exp_fast(t.m - m);
        t.u = e * (t.u + t.s * d);
        t.s *= e;
        t.m = m;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = z[i] - m, e = exp_fast(d);
        t.s += e;
        t.u = fmaf(e, fmaxf(d, kFar), t.u);
    }
}

struct Args {
    const void *z;
    int64_t class_stride, token_stride, V, B;
    const int64_t *targets;
    int64_t top;
    float *logprob, *entropy, *lse, *top_logprob;
    int64_t *top_index;
    float4 *parts;                      // [B][nparts] Stat of each part
    float *maxima;                      // [B][nseg], kept if top > 0
    int64_t nparts, nseg, part_len, seg_len;
    int64_t first;                      // the launch's first row or tile
};

// ---- the k greatest -------------------------------------------------------------------

// A float's place in the order of logits: NaN first, +0 and -0 alike.
__device__ __forceinline__ uint32_t order_of(float z) {
    if (z != z) return ~0u;
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The k greatest 64-bit keys seen so far, one per lane in descending order (0 = none).
struct TopList {
    uint64_t key = 0;
    __device__ __forceinline__ uint64_t least(int k) const {
        return uint64_t(__shfl(static_cast<unsigned long long>(key), k - 1, kWave));
    }
    // every lane offers a key (0 = none); all lanes take part
    __device__ __forceinline__ void offer(uint64_t mine, int k, int lane) {
        uint64_t floor = least(k);
        uint64_t who = __ballot(mine > floor);
        while (who) {
            const int src = __ffsll(static_cast<unsigned long long>(who)) - 1;
            const uint64_t c = __shfl(static_cast<unsigned long long>(mine), src, kWave);
            const uint64_t up = __shfl_up(static_cast<unsigned long long>(key), 1, kWave);
            const int at = __popcll(__ballot(key > c));          // keys are distinct
            key = lane < at ? key : lane == at ? c : up;
            floor = least(k);
            if (lane == src) mine = 0;
            who = __ballot(mine > floor);
        }
    }
};

// One wave: the alternatives of token b, given the segments' maxima.
template <typename T>
__device__ __forceinline__ void write_top(const Args &a, int64_t b, const float *maxima, float lse,
                                          int lane) {
    const int k = int(a.top);
    TopList segs;
    for (int64_t i = 0; i < a.nseg; i += kWave) {
        const int64_t s = i + lane;
        const uint64_t key = s < a.nseg ? uint64_t(order_of(maxima[s])) << 32 | (UINT32_MAX - uint32_t(s)) : 0;
        segs.offer(key, k, lane);
    }
    const T *col = static_cast<const T *>(a.z) + b * a.token_stride;
    TopList best;
    for (int i = 0; i < k; ++i) {
        const uint64_t key = __shfl(static_cast<unsigned long long>(segs.key), i, kWave);
        if (key == 0) break;
        const int64_t first = int64_t(UINT32_MAX - uint32_t(key)) * a.seg_len;
        int64_t last = first + a.seg_len;
        if (last > a.V) last = a.V;
        for (int64_t v0 = first; v0 < last; v0 += kWave) {
            const int64_t v = v0 + lane;
            uint64_t mine = 0;
            if (v < last)
                mine = uint64_t(order_of(float(col[v * a.class_stride]))) << 32 | (UINT32_MAX - uint32_t(v));
            best.offer(mine, k, lane);
        }
    }
    if (lane < k) {
        const int64_t v = UINT32_MAX - uint32_t(best.key);
        const float z = float(col[v * a.class_stride]);
        a.top_index[b * a.top + lane] = v;
        a.top_logprob[b * a.top + lane] = lse == -kInf ? -kInf : z - lse;
    }
}

// One wave: a token's results from its whole Stat.
template <typename T>
__device__ __forceinline__ float write_token(const Args &a, int64_t b, Stat t, int lane) {
    const bool empty = t.m == -kInf && t.s == 0.0f;         // nothing but -inf
    const float logs = logf(t.s), lse = empty ? -kInf : t.m + logs;
    if (lane == 0) {
        const int64_t y = a.targets ? a.targets[b] : -1;
        float lp = 0.0f;
        if (y >= a.V) {
            lp = __builtin_nanf("");
        } else if (y >= 0) {
            const float z = float(static_cast<const T *>(a.z)[b * a.token_stride + y * a.class_stride]);
            lp = empty ? -kInf : z - lse;
        }
        a.logprob[b] = lp;
        a.entropy[b] = empty ? 0.0f : logs - t.u / t.s;
        a.lse[b] = lse;
    }
    return lse;
}

// ---- token-major: a row's classes are contiguous --------------------------------------

// grid (parts, B); each wave takes every kWaves-th run of 64 vectors of its part, which is a
// segment: its maximum is also what the wave's sums run from.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(Args a) {
    constexpr int V = kVec<T>, kWaves = kRowThreads / kWave, kRun = V * kWave;
    __shared__ Stat stats[kWaves];
    const int w = threadIdx.x / kWave, lane = lane_id();
    const int64_t b = a.first + blockIdx.y, part = blockIdx.x;
    const T *row = static_cast<const T *>(a.z) + b * a.token_stride;
    const int64_t begin = part * a.part_len;
    int64_t end = begin + a.part_len;
    if (end > a.V) end = a.V;
    Stat t{-kInf, 0.0f, 0.0f};
    for (int64_t v0 = begin + w * kRun; v0 < end; v0 += kWaves * kRun) {
        const int64_t v = v0 + lane * V;
        float z[V];
        if (v + V <= end) {
            const Loaded<T, V> x = load_vec<T, V>(row + v);
#pragma unroll
            for (int i = 0; i < V; ++i) z[i] = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) z[i] = v + i < end ? float(row[v + i]) : -kInf;
        }
        float m = z[0];
        bool nan = z[0] != z[0];
#pragma unroll
        for (int i = 1; i < V; ++i) {
            m = fmaxf(m, z[i]);
            nan |= z[i] != z[i];
        }
        nan = __any(nan);
        m = wave_max(m);
        if (a.top && lane == 0) a.maxima[b * a.nseg + v0 / kRun] = nan ? __builtin_nanf("") : m;
        add_values(t, z, fmaxf(m, t.m));
        if (nan) t.s = __builtin_nanf("");
    }
    for (int d = 1; d < kWave; d <<= 1) t = join(t, shuffle_xor(t, d));
    if (lane == 0) stats[w] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kWaves; ++i) t = join(t, stats[i]);
        a.parts[b * a.nparts + part] = make_float4(t.m, t.s, t.u, 0.0f);
    }
}

// ---- feature-major: a class's tokens are contiguous -----------------------------------

// grid (parts, token tiles of kLanes * V): a lane takes V tokens, kLanes of them a row of the
// tile; a thread takes runs of kColRun classes, each a segment.  Tokens past the end: the last
// V again (the same values are written twice).
template <typename T, int V, int kLanes>
__global__ __launch_bounds__(kColThreads) void columns_kernel(Args a) {
    constexpr int kRows = kColThreads / kLanes;
    __shared__ float sm[kRows][kLanes * V], ss[kRows][kLanes * V], su[kRows][kLanes * V];
    const int tx = threadIdx.x % kLanes, ty = threadIdx.x / kLanes;
    const int64_t part = blockIdx.x, tile = a.first + blockIdx.y;
    int64_t b = (tile * kLanes + tx) * V;
    const bool live = b < a.B;
    if (b > a.B - V) b = a.B - V;
    const T *z = static_cast<const T *>(a.z) + b;
    const int64_t begin = part * a.part_len;
    int64_t end = begin + a.part_len;
    if (end > a.V) end = a.V;
    Stat t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = {-kInf, 0.0f, 0.0f};
    for (int64_t v0 = begin + ty * kColRun; v0 < end; v0 += kRows * kColRun) {
        float m[V];
        bool nan[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            m[j] = -kInf;
            nan[j] = false;
        }
        constexpr int kAtOnce = 8;
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
                    nan[j] |= y[r] != y[r];
                }
                m[j] = top;
                add_values(t[j], y, fmaxf(top, t[j].m));
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (nan[j]) t[j].s = __builtin_nanf("");
            if (a.top && live) a.maxima[(b + j) * a.nseg + v0 / kColRun] = nan[j] ? __builtin_nanf("") : m[j];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        sm[ty][tx * V + j] = t[j].m;
        ss[ty][tx * V + j] = t[j].s;
        su[ty][tx * V + j] = t[j].u;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kLanes * V; i += kColThreads) {
        Stat all{sm[0][i], ss[0][i], su[0][i]};
        for (int r = 1; r < kRows; ++r) all = join(all, {sm[r][i], ss[r][i], su[r][i]});
        // where lane i / V has its tokens
        const int64_t own = (tile * kLanes + i / V) * V;
        if (own < a.B)
            a.parts[((own > a.B - V ? a.B - V : own) + i % V) * a.nparts + part] =
                make_float4(all.m, all.s, all.u, 0.0f);
    }
}

// A wave per token: its parts joined, the results written, the alternatives found.
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(Args a) {
    const int lane = lane_id();
    const int64_t b = int64_t(blockIdx.x) * (kJoinThreads / kWave) + threadIdx.x / kWave;
    if (b >= a.B) return;
    Stat t{-kInf, 0.0f, 0.0f};
    for (int64_t i = lane; i < a.nparts; i += kWave) {
        const float4 p = a.parts[b * a.nparts + i];
        t = join(t, {p.x, p.y, p.z});
    }
    for (int d = 1; d < kWave; d <<= 1) t = join(t, shuffle_xor(t, d));
    const float lse = write_token<T>(a, b, t, lane);
    if (a.top) write_top<T>(a, b, a.maxima + b * a.nseg, lse, lane);
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
    int64_t target;
};

__device__ __forceinline__ Column column_of(const GradArgs &a, int64_t b) {
    Column c;
    c.lse = a.lse[b];
    c.target = a.targets ? a.targets[b] : -1;
    c.g = a.grad_logprob ? a.grad_logprob[b] : 0.0f;
    c.ge = a.grad_entropy ? a.grad_entropy[b] : 0.0f;
    c.h = a.grad_entropy ? a.entropy[b] : 0.0f;
    if (c.target < 0) c.g = 0.0f;                    // no given token
    if (c.target >= a.V) c.g = __builtin_nanf("");   // no such token
    if (c.lse == -kInf) {                            // nothing but -inf: no gradient
        c.lse = c.g = c.ge = c.h = 0.0f;
    }
    return c;
}

// p (-g - ge (log p + H)), and g more at the given token; zero where p is.
template <bool ENTROPY>
__device__ __forceinline__ float gradient(const Column &c, float z, int64_t v) {
    const float lp = z - c.lse, p = exp_fast(lp);
    float f = -c.g;
    if (ENTROPY) f -= c.ge * (fmaxf(lp, kFar) + c.h);
    const float d = p * f;
    return v == c.target ? d + c.g : d;
}

constexpr int kGradThreads = 256;

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
            for (int j = 0; j < V; ++j) d[j] = gradient<ENTROPY>(c, x[i][j], v + j);
            store_vec<T, V>(dz + v, d);
        } else {
            for (int64_t k = v; k < a.V; ++k) dz[k] = T(gradient<ENTROPY>(c, float(z[k]), k));
        }
    }
}

// Feature-major: grid (class parts, token tiles); a thread takes V tokens of kEach classes.
// The last lane's tokens start where a whole vector fits; what the lane before it writes too
// it leaves out, since dz may be z.
template <typename T, int V, int kLanes, bool ENTROPY>
__global__ __launch_bounds__(kGradThreads) void grad_columns_kernel(GradArgs a) {
    constexpr int kRows = kGradThreads / kLanes, kEach = 8;
    const int tx = threadIdx.x % kLanes, ty = threadIdx.x / kLanes;
    const int64_t b = ((a.first + blockIdx.y) * kLanes + tx) * V;
    if (b >= a.B) return;
    const int n = a.B - b < V ? int(a.B - b) : V;
    const T *z = static_cast<const T *>(a.z) + b;
    T *dz = static_cast<T *>(a.dz) + b;
    Column c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = column_of(a, b + (j < n ? j : 0));
    const int64_t v0 = int64_t(blockIdx.x) * (kRows * kEach) + ty;
    if (n == V) {
        Loaded<T, V> x[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t v = v0 + i * kRows;
            x[i] = load_vec<T, V>(z + (v < a.V ? v : a.V - 1) * a.class_stride);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t v = v0 + i * kRows;
            if (v >= a.V) break;
            float d[V];
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = gradient<ENTROPY>(c[j], x[i][j], v);
            store_vec<T, V>(dz + v * a.out_class_stride, d);
        }
    } else {
        for (int i = 0; i < kEach; ++i) {
            const int64_t v = v0 + i * kRows;
            if (v >= a.V) break;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < n)
                    dz[v * a.out_class_stride + j] =
                        T(gradient<ENTROPY>(c[j], float(z[v * a.class_stride + j]), v));
        }
    }
}

constexpr int64_t kMaxGridY = 65535;

// One launch per 65535 rows or tiles.
template <typename A, typename F> hipError_t over_grid_y(A a, int64_t n, F &&launch) {
    for (a.first = 0; a.first < n; a.first += kMaxGridY) {
        launch(a, unsigned(n - a.first < kMaxGridY ? n - a.first : kMaxGridY));
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
    int64_t part_len, nparts, seg_len, nseg;
};

Cut cut_of(int dtype, int64_t V, int64_t B, bool rows) {
    Cut c;
    c.rows = rows;
    c.vec = dtype == DARB_F32 ? 4 : 8;
    if (rows) {
        c.lanes = 0;
        c.seg_len = c.vec * kWave;
        const int64_t step = c.seg_len * (kRowThreads / kWave);     // one round of a workgroup
        const int64_t rounds = (V + step - 1) / step;
        // about 1024 workgroups, each of at least 4 rounds
        int64_t parts = (1024 + B - 1) / B;
        if (parts > rounds / 4) parts = rounds / 4;
        if (parts < 1) parts = 1;
        c.part_len = (rounds + parts - 1) / parts * step;
    } else {
        if (B < c.vec) c.vec = 1;
        c.lanes = lanes_of(B, c.vec);
        c.seg_len = kColRun;
        const int64_t step = kColThreads / c.lanes * kColRun;       // one round of a workgroup
        const int64_t rounds = (V + step - 1) / step;
        const int64_t tiles = (B + c.lanes * c.vec - 1) / (c.lanes * c.vec);
        int64_t parts = (1024 + tiles - 1) / tiles;
        if (parts > rounds) parts = rounds;
        c.part_len = (rounds + parts - 1) / parts * step;
    }
    c.nparts = (V + c.part_len - 1) / c.part_len;
    c.nseg = (V + c.seg_len - 1) / c.seg_len;
    return c;
}

// Either order of the logits has its class or its token stride 1 (with one class or one token
// the other stride is never used).
bool rows_of(int64_t V, int64_t class_stride) { return V == 1 || class_stride == 1; }

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

int64_t logprobs_max_top() { return kMaxTop; }

// Enough for either order and every type.
int64_t logprobs_workspace_bytes(int64_t V, int64_t B, int64_t top) {
    int64_t parts = 0;
    for (int dtype : {int(DARB_F32), int(DARB_F16)})
        for (bool rows : {false, true}) {
            const Cut c = cut_of(dtype, V, B, rows);
            if (c.nparts > parts) parts = c.nparts;
        }
    return padded(parts * B * 16) + (top ? padded((V + kColRun - 1) / kColRun * B * 4) : 0);
}

hipError_t launch_logprobs(int dtype, int64_t V, int64_t B, const void *z, int64_t class_stride,
                           int64_t token_stride, const int64_t *targets, int64_t top,
                           float *logprob, float *entropy, float *lse, float *top_logprob,
                           int64_t *top_index, void *workspace, hipStream_t s) {
    const Cut c = cut_of(dtype, V, B, rows_of(V, class_stride));
    float *maxima = reinterpret_cast<float *>(static_cast<char *>(workspace) + padded(c.nparts * B * 16));
    const Args a{z, class_stride, token_stride, V, B, targets, top, logprob, entropy, lse,
                 top_logprob, top_index, static_cast<float4 *>(workspace), maxima, c.nparts,
                 c.nseg, c.part_len, c.seg_len, 0};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        hipError_t e;
        if (c.rows) {
            e = over_grid_y(a, B, [&](const Args &part, unsigned n) {
                hipLaunchKernelGGL((rows_kernel<T>), dim3(unsigned(c.nparts), n),
                                   dim3(kRowThreads), 0, s, part);
            });
        } else {
            const int64_t tiles = (B + c.lanes * c.vec - 1) / (c.lanes * c.vec);
            auto columns = [&](auto vec) {
                constexpr int V1 = decltype(vec)::value;
                return with_lanes<V1>(c.lanes, [&](auto lanes) {
                    constexpr int L = decltype(lanes)::value;
                    return over_grid_y(a, tiles, [&](const Args &part, unsigned n) {
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
        const int64_t waves = kJoinThreads / kWave;
        hipLaunchKernelGGL((join_kernel<T>), dim3(unsigned((B + waves - 1) / waves)),
                           dim3(kJoinThreads), 0, s, a);
        return hipGetLastError();
    });
}

hipError_t launch_logprobs_grad(int dtype, int64_t V, int64_t B, const void *z,
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
            if (rows_of(V, class_stride)) {
                const int64_t each = kGradThreads * 4 * VT;
                return over_grid_y(a, B, [&](const GradArgs &part, unsigned n) {
                    hipLaunchKernelGGL((grad_rows_kernel<T, E>),
                                       dim3(unsigned((V + each - 1) / each), n),
                                       dim3(kGradThreads), 0, s, part);
                });
            }
            const int lanes = lanes_of(B, VT);
            const int64_t tiles = (B + lanes * VT - 1) / (lanes * VT);
            const int64_t each = kGradThreads / lanes * 8;
            return with_lanes<VT>(lanes, [&](auto l) {
                constexpr int L = decltype(l)::value;
                return over_grid_y(a, tiles, [&](const GradArgs &part, unsigned n) {
                    hipLaunchKernelGGL((grad_columns_kernel<T, VT, L, E>),
                                       dim3(unsigned((V + each - 1) / each), n),
                                       dim3(kGradThreads), 0, s, part);
                });
            });
        };
        return grad_entropy ? launch(std::true_type{}) : launch(std::false_type{});
    });
}

}  // namespace darb
