// Layer norm of the columns of x [H x B] and its gradients.
//
//   mean = sum_h x / H,  rstd = 1 / sqrt(sum_h (x - mean)^2 / H + eps),
//   xh = (x - mean) rstd,  y = xh w + b
//   a = dy w,  dx = rstd (a - sum_h a / H - xh sum_h a xh / H)
//   dw = sum_b dy xh,  db = sum_b dy
//
// Memory-bound: a column is read once into registers, where its sums run twice over it (the
// variance around the mean itself, not from a difference of sums).  dw and db run over all
// columns: each workgroup sums the columns it takes, rows of partial sums go to the workspace,
// and a last launch adds them in a fixed order.
//
// Measured on MI355X, among other calls: forward 1024 x 32 fp32 6.6 us (latency of one round of
// loads and two sums), 4096 x 4096 27 (4.9 TB/s); gradients of 1024 x 6400 fp32 feature-major
// 25.8 (3.1 TB/s: all loads, then the sums, then all stores), of 9216 x 2047 token-major bf16 35.4
// (3.2 TB/s; partial rows are a sixth of it) and fp32 54 (4.2 TB/s; 43 out of the cache); forward of
// the same bf16 16.4 (4.6 TB/s).
#include <type_traits>

#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxWaves = kMaxThreads / kWave;
constexpr int kGradThreads = 512;       // twice the registers a thread: x, dy and the sums
// Feature-major gradients: fp32 tiles of whole cache lines in workgroups of 1024 threads; the
// sums of 8 tokens a lane need the registers of 512.
template <typename T> constexpr int kTileThreads = sizeof(T) == 4 ? 1024 : kGradThreads;
template <typename T> constexpr int kMostHeld = sizeof(T) == 4 ? 8 : 16;

struct Matrix {                         // element (h, b) at h * feature + b * token
    void *p;
    int64_t feature, token;
};

struct Args {
    Matrix x, y, dy;                    // y: y, or dx
    const void *w, *b;
    int w_f32;                          // w and b are fp32 (else of x's type)
    int64_t H, B;
    float eps;
    float *mean, *rstd;
    float *dw, *db;                     // partial sums [blocks][H], or null
    int64_t first;                      // the launch's first token or tile
};

template <typename T>
__device__ __forceinline__ float weight_at(const Args &a, const void *w, int64_t h) {
    return a.w_f32 ? static_cast<const float *>(w)[h] : float(static_cast<const T *>(w)[h]);
}

// V weights from feature h on; `none` where there are no weights.
template <typename T, int V>
__device__ __forceinline__ void weights(const Args &a, const void *w, int64_t h, float none,
                                        float (&f)[V]) {
    if (!w) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = none;
    } else if (a.w_f32) {
        const Loaded<float, V> x = load_vec<float, V>(static_cast<const float *>(w) + h);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = x[j];
    } else {
        const Loaded<T, V> x = load_vec<T, V>(static_cast<const T *>(w) + h);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = x[j];
    }
}

// The sum of s[0 .. N) over `waves` waves of the workgroup from `first` on, each in every thread;
// scratch: N * kMaxWaves floats.
template <int N>
__device__ __forceinline__ void block_sum(float (&s)[N], float *scratch, int first, int waves) {
    const int w = wave_id();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if (blockDim.x == kWave) return;
    __syncthreads();                                 // the scratch's last use
    if (lane_id() == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) scratch[i * kMaxWaves + w] = s[i];
    __syncthreads();
    // a lane reads one wave's sum: one latency for all of them
    const int k = lane_id() % kMaxWaves;
#pragma unroll
    for (int i = 0; i < N; ++i)
        s[i] = lane_of(group_reduce<kMaxWaves, AddOp>(k < waves ? scratch[i * kMaxWaves + first + k] : 0.0f), kMaxWaves - 1);
}

// A vector that would pass the end of its axis starts V before it instead, and leaves out its
// first `skip` elements, which belong to others: no access is partial or divergent but the last
// vector's store.
template <int V> __device__ __forceinline__ int64_t back_from_end(int64_t at, int64_t end, int &skip) {
    const int64_t own = at + V <= end ? at : end - V;
    skip = at - own < V ? int(at - own) : V;
    return own;
}

template <typename T, int V> __device__ __forceinline__ void store_own(T *p, int skip, const float (&f)[V]) {
    if (skip == 0) {
        store_vec<T, V>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= skip) p[i] = T(f[i]);
    }
}

// ---- token-major: a token's features are contiguous -----------------------------------
//
// A workgroup per token; a thread holds N vectors of the row, a workgroup's width apart.  N = 0:
// a row longer than the registers of 1024 threads, read again for every sum.

template <typename T, int V, int N> struct Row {
    Loaded<T, V> held[N ? N : 1];
    const T *p;
    int64_t H;
    int tid, threads;                   // the thread's place among a row's

    // f(vector's place in the thread, its first feature, elements to leave out, vector)
    template <typename F> __device__ __forceinline__ void each(F &&f) const {
        int skip;
        if constexpr (N) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t at = (int64_t(i) * threads + tid) * V;
                if (at >= H) break;
                const int64_t h = back_from_end<V>(at, H, skip);
                f(i, h, skip, held[i]);
            }
        } else {
            for (int64_t at = int64_t(tid) * V; at < H; at += int64_t(threads) * V) {
                const int64_t h = back_from_end<V>(at, H, skip);
                f(0, h, skip, load_vec<T, V>(p + h));
            }
        }
    }
    __device__ __forceinline__ void forget() {
        if constexpr (N) {
#pragma unroll
            for (int i = 0; i < N; ++i) forget_uses(held[i]);
        }
    }
    __device__ __forceinline__ void open(const T *row, int64_t len, int tid_, int threads_) {
        p = row;
        H = len;
        tid = tid_;
        threads = threads_;
        if constexpr (N) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int skip;
                const int64_t at = (int64_t(i) * threads + tid) * V;
                held[i] = load_vec<T, V>(p + back_from_end<V>(at, H, skip));
            }
        }
    }
};

template <typename T, int V, int N>
__global__ __launch_bounds__(kMaxThreads) void norm_rows_kernel(Args a) {
    __shared__ float scratch[kMaxWaves];
    const int64_t b = a.first + blockIdx.x;
    Row<T, V, N> x;
    x.open(static_cast<const T *>(a.x.p) + b * a.x.token, a.H, threadIdx.x, blockDim.x);
    T *y = static_cast<T *>(a.y.p) + b * a.y.token;
    float s[1] = {0.0f};
    x.each([&](int, int64_t, int skip, const Loaded<T, V> &v) {
#pragma unroll
        for (int j = 0; j < V; ++j) s[0] += j >= skip ? v[j] : 0.0f;
    });
    block_sum(s, scratch, 0, blockDim.x / kWave);
    x.forget();
    const float mean = s[0] / float(a.H);
    s[0] = 0.0f;
    x.each([&](int, int64_t, int skip, const Loaded<T, V> &v) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = j >= skip ? v[j] - mean : 0.0f;
            s[0] = fmaf(d, d, s[0]);
        }
    });
    block_sum(s, scratch, 0, blockDim.x / kWave);
    x.forget();
    const float rstd = 1.0f / sqrtf(s[0] / float(a.H) + a.eps);
    x.each([&](int, int64_t h, int skip, const Loaded<T, V> &v) {
        float w[V], c[V], out[V];
        weights<T, V>(a, a.w, h, 1.0f, w);
        weights<T, V>(a, a.b, h, 0.0f, c);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = fmaf((v[j] - mean) * rstd, w[j], c[j]);
        store_own<T, V>(y + h, skip, out);
    });
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[b] = mean;
        if (a.rstd) a.rstd[b] = rstd;
    }
}

// Threads of a workgroup whose registers (128 or 256 a thread) hold n vectors of two rows, this
// one and the next, and their sums without spilling.
constexpr int row_threads(int vec, int n) { return n > 0 && n * (vec + 4) <= 24 ? kMaxThreads : kGradThreads; }

// A workgroup is one or several teams of `threads` threads, each of which takes a token at a
// time: teams of one wave (WAVES) without a barrier, larger ones in step.  (One row of 1500 at a
// time left a CU's SIMDs waiting: 8192 of them in bf16 took 47 us, four together 26.)  Held rows:
// dw and db sum in registers, the teams' then in LDS; longer ones: in the workgroup's row of the
// workspace.
template <typename T, int V, int N, bool WAVES>
__global__ __launch_bounds__(WAVES ? kGradThreads : row_threads(V, N)) void norm_grad_rows_kernel(
    Args a, int threads) {
    constexpr int kHeld = N ? N : 1;
    constexpr bool kSeveral = WAVES || row_threads(V, N) > kGradThreads;
    __shared__ float scratch[2 * kMaxWaves];
    if (WAVES) threads = kWave;
    const int waves = threads / kWave;                             // of a row
    const int team = kSeveral ? wave_id() / waves : 0, teams = kSeveral ? int(blockDim.x) / threads : 1;
    const int tid = threadIdx.x - team * threads;
    const int64_t step = int64_t(gridDim.x) * teams, first_b = int64_t(blockIdx.x) * teams + team;
    float *dw = a.dw ? a.dw + blockIdx.x * a.H : nullptr;
    float *db = a.db ? a.db + blockIdx.x * a.H : nullptr;
    float sw[kHeld][V], sb[kHeld][V];
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) sw[i][j] = sb[i][j] = 0.0f;
    // The next token's rows are on their way while this one's sums cross the workgroup.  Loads
    // return in order: nothing that is needed sooner may be issued after them.
    float held_w[kHeld][V];
    if constexpr (N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int skip;
            const int64_t at = (int64_t(i) * threads + tid) * V;
            weights<T, V>(a, a.w, back_from_end<V>(at, a.H, skip), 1.0f, held_w[i]);
        }
    }
    Row<T, V, N> next_x, next_dy;
    float next_mean, next_rstd;
    auto fetch = [&](int64_t b) {
        next_mean = a.mean[b];
        next_rstd = a.rstd[b];
        next_x.open(static_cast<const T *>(a.x.p) + b * a.x.token, a.H, tid, threads);
        next_dy.open(static_cast<const T *>(a.dy.p) + b * a.dy.token, a.H, tid, threads);
    };
    if (first_b < a.B) fetch(first_b);
    for (int64_t b = first_b; b - team < a.B; b += step) {          // as often in every team
        const bool live = !kSeveral || b < a.B;
        Row<T, V, N> x = next_x, dy = next_dy;
        const float mean = next_mean, rstd = next_rstd;
        if (b + step < a.B) fetch(b + step);
        T *dx = static_cast<T *>(a.y.p) + b * a.y.token;
        float s[2] = {0.0f, 0.0f};
        if (live) x.each([&](int i, int64_t h, int skip, const Loaded<T, V> &v) {
            const Loaded<T, V> g = N ? dy.held[i] : load_vec<T, V>(dy.p + h);
            float w[V];
            if constexpr (N) {
#pragma unroll
                for (int j = 0; j < V; ++j) w[j] = held_w[i][j];
            } else {
                weights<T, V>(a, a.w, h, 1.0f, w);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool own = j >= skip;
                const float gj = own ? g[j] : 0.0f, xh = own ? (v[j] - mean) * rstd : 0.0f;
                const float c = gj * w[j];
                s[0] += c;
                s[1] = fmaf(c, xh, s[1]);
                if constexpr (N) {
                    sw[i][j] = fmaf(gj, xh, sw[i][j]);
                    sb[i][j] += gj;
                } else if (own) {
                    const bool first = b == blockIdx.x;
                    if (dw) dw[h + j] = first ? gj * xh : fmaf(gj, xh, dw[h + j]);
                    if (db) db[h + j] = first ? gj : db[h + j] + gj;
                }
            }
        });
        if (!a.y.p) continue;
        if constexpr (WAVES) {
            s[0] = wave_sum(s[0]);
            s[1] = wave_sum(s[1]);
        } else {
            block_sum(s, scratch, team * waves, waves);
        }
        if (!live) continue;                         // the last round
        x.forget();
        dy.forget();
        const float m0 = s[0] / float(a.H), m1 = s[1] / float(a.H);
        x.each([&](int i, int64_t h, int skip, const Loaded<T, V> &v) {
            const Loaded<T, V> g = N ? dy.held[i] : load_vec<T, V>(dy.p + h);
            float w[V], out[V];
            if constexpr (N) {
#pragma unroll
                for (int j = 0; j < V; ++j) w[j] = held_w[i][j];
            } else {
                weights<T, V>(a, a.w, h, 1.0f, w);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (v[j] - mean) * rstd;
                out[j] = rstd * (g[j] * w[j] - m0 - xh * m1);
            }
            store_own<T, V>(dx + h, skip, out);
        });
    }
    if constexpr (N) {
        // team by team, in LDS; the last one's sums are the workgroup's
        __shared__ float together[kSeveral ? N * V * (WAVES ? kWave : kGradThreads) : 1];
        auto add = [&](float (&sum)[kHeld][V]) {
            for (int turn = 0; turn < teams && teams > 1; ++turn) {
                if (team == turn) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            float &t = together[(i * V + j) * threads + tid];
                            if (turn > 0) sum[i][j] += t;
                            t = sum[i][j];
                        }
                }
                __syncthreads();
            }
        };
        if constexpr (kSeveral) {
            add(sw);
            add(sb);
        }
        if (team + 1 < teams) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = (int64_t(i) * threads + tid) * V;
            if (at >= a.H) break;
            int skip;
            const int64_t h = back_from_end<V>(at, a.H, skip);
            if (dw) store_own<float, V>(dw + h, skip, sw[i]);
            if (db) store_own<float, V>(db + h, skip, sb[i]);
        }
    }
}

// ---- feature-major: a feature's tokens are contiguous ---------------------------------
//
// A workgroup takes a tile of `lanes` * V tokens: a thread V tokens of every rows-th feature,
// N of them in registers.  N = 0: more features than that, read again for every sum.

template <typename T, int V, int N> struct Tile {
    Loaded<T, V> held[N ? N : 1];
    const T *p;
    int64_t H, stride;
    uint32_t at;                        // the thread's first vector, in bytes from p
    int first, rows;

    // a vector of feature i * rows + first: a base that the workgroup shares and 32 bits of a
    // thread's own (tile_shape sees to it that they suffice where N is not 0)
    __device__ __forceinline__ const T *row(int64_t i) const {
        return reinterpret_cast<const T *>(reinterpret_cast<const char *>(p + i * rows * stride) + at);
    }
    // f(feature's place in the thread, feature, vector)
    template <typename F> __device__ __forceinline__ void each(F &&f) const {
        if constexpr (N) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t h = first + int64_t(i) * rows;
                if (h < H) f(i, h, held[i]);
            }
        } else {
            for (int64_t h = first; h < H; h += rows) f(0, h, get(h));
        }
    }
    __device__ __forceinline__ Loaded<T, V> get(int64_t h) const {
        return load_vec<T, V>(p + b + h * stride);
    }
    __device__ __forceinline__ void forget() {
        if constexpr (N) {
#pragma unroll
            for (int i = 0; i < N; ++i) forget_uses(held[i]);
        }
    }
    int64_t b;
    __device__ __forceinline__ void open(const void *p_, int64_t b_, int64_t H_, int64_t stride_, int first_, int rows_) {
        p = static_cast<const T *>(p_);
        b = b_;
        H = H_;
        stride = stride_;
        first = first_;
        rows = rows_;
        if constexpr (N) {
            // past the last feature: the thread's tokens of the round's first one
            const uint32_t token = uint32_t(b) * uint32_t(sizeof(T));
            const uint32_t own = token + uint32_t(first) * uint32_t(stride) * uint32_t(sizeof(T));
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (int64_t(i) * rows >= H) break;
                at = first + int64_t(i) * rows < H ? own : token;
                held[i] = load_vec<T, V>(row(i));
            }
            at = own;
        }
    }
};

template <typename T, int V, int N>
__device__ __forceinline__ T *out_row(const Matrix &m, int64_t i, int64_t h, int first, int rows, int64_t b) {
    if constexpr (N) {
        const uint32_t at = (uint32_t(first) * uint32_t(m.feature) + uint32_t(b)) * uint32_t(sizeof(T));
        return reinterpret_cast<T *>(reinterpret_cast<char *>(static_cast<T *>(m.p) + i * rows * m.feature) + at);
    } else {
        return static_cast<T *>(m.p) + b + h * m.feature;
    }
}

// x summed over the lanes of a wave that are equal modulo `lanes` (1, 2, 4 or 8): rotations
// inside rows of 16, then across the rows.  (Lanes add in different orders.)
__device__ __forceinline__ float sum_equal_lanes(float x, int lanes) {
    constexpr int kRor8 = 0x128, kRor4 = 0x124;
    if (lanes <= 1) x += dpp_all<kDppXor1>(x);
    if (lanes <= 2) x += dpp_all<kDppXor2>(x);
    if (lanes <= 4) x += dpp_all<kRor4>(x);
    x += dpp_all<kRor8>(x);
    return sum_rows(x);
}

constexpr int kMaxLanes = 8;

// What tile_sum needs for K sums of up to kMaxLanes lanes.
template <int K> struct TileRoom {
    float waves[K * kMaxLanes * kMaxWaves], sums[K * kMaxLanes];
};

// s summed over the threads with the same tokens (lanes of them side by side), in each of them.
// The waves' sums are added by a row of 16 lanes each, one wave's sum a lane: read by every
// thread, one after the other, they took a fifth of a small call.
template <int K> __device__ __forceinline__ void tile_sum(float (&s)[K], int lanes, TileRoom<K> &room) {
    const int waves = blockDim.x / kWave, w = wave_id(), lane = lane_id();
#pragma unroll
    for (int j = 0; j < K; ++j) s[j] = sum_equal_lanes(s[j], lanes);
    if (lane < lanes)                                // the room's last use is two barriers ago
#pragma unroll
        for (int j = 0; j < K; ++j) room.waves[(j * lanes + lane) * kMaxWaves + w] = s[j];
    __syncthreads();
    for (int i = threadIdx.x; i < K * lanes * kMaxWaves; i += blockDim.x) {      // whole rows
        const int k = i % kMaxWaves;
        const float sum = group_reduce<kMaxWaves, AddOp>(k < waves ? room.waves[i] : 0.0f);
        if (k == kMaxWaves - 1) room.sums[i / kMaxWaves] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < K; ++j) s[j] = room.sums[j * lanes + (lane & (lanes - 1))];
}

__device__ __forceinline__ int log2_of(int power) { return __ffs(power) - 1; }

// The tile of task i: tasks go to the 8 XCDs in turn, each with an L2 of its own, and tiles that
// lie side by side (parts of the same cache lines, where a tile is narrow) go to one XCD.
__device__ __forceinline__ int64_t tile_of(int64_t i, int64_t tiles) {
    const int64_t xcd = i % 8, whole = tiles / 8, more = tiles % 8;
    return xcd * whole + (xcd < more ? xcd : more) + i / 8;
}

template <typename T, int V, int N>
__global__ __launch_bounds__(kMaxThreads) void norm_columns_kernel(Args a, int lanes) {
    constexpr int kHeld = N < 16 ? N : 0;            // weights: with 16 vectors they would spill
    __shared__ TileRoom<V> room;
    const int tx = threadIdx.x & (lanes - 1), ty = threadIdx.x >> log2_of(lanes), rows = blockDim.x >> log2_of(lanes);
    int skip;
    const int64_t b = back_from_end<V>(((a.first + tile_of(blockIdx.x, gridDim.x)) * lanes + tx) * V, a.B, skip);
    float w[kHeld ? kHeld : 1], c[kHeld ? kHeld : 1];
    if constexpr (kHeld) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int64_t h = ty + int64_t(i) * rows < a.H ? ty + int64_t(i) * rows : 0;
            w[i] = a.w ? weight_at<T>(a, a.w, h) : 1.0f;
            c[i] = a.b ? weight_at<T>(a, a.b, h) : 0.0f;
        }
    }
    Tile<T, V, N> x;
    x.open(a.x.p, b, a.H, a.x.feature, ty, rows);
    float mean[V], rstd[V];
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] = rstd[j] = 0.0f;
    x.each([&](int, int64_t, const Loaded<T, V> &v) {
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] += v[j];
    });
    tile_sum(mean, lanes, room);
    x.forget();
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] /= float(a.H);
    x.each([&](int, int64_t, const Loaded<T, V> &v) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = v[j] - mean[j];
            rstd[j] = fmaf(d, d, rstd[j]);
        }
    });
    tile_sum(rstd, lanes, room);
    x.forget();
#pragma unroll
    for (int j = 0; j < V; ++j) rstd[j] = 1.0f / sqrtf(rstd[j] / float(a.H) + a.eps);
    x.each([&](int i, int64_t h, const Loaded<T, V> &v) {
        float wh, ch, out[V];
        if constexpr (kHeld) {
            wh = w[i];
            ch = c[i];
        } else {
            wh = a.w ? weight_at<T>(a, a.w, h) : 1.0f;
            ch = a.b ? weight_at<T>(a, a.b, h) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = fmaf((v[j] - mean[j]) * rstd[j], wh, ch);
        store_own<T, V>(out_row<T, V, N>(a.y, i, h, ty, rows, b), skip, out);
    });
    if (ty == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (j >= skip && a.mean) a.mean[b + j] = mean[j];
            if (j >= skip && a.rstd) a.rstd[b + j] = rstd[j];
        }
    }
}

template <typename T, int V, int N>
__global__ __launch_bounds__(kTileThreads<T>) void norm_grad_columns_kernel(Args a, int lanes) {
    constexpr int kHeld = N ? N : 1;
    __shared__ TileRoom<2 * V> room;
    const int tx = threadIdx.x & (lanes - 1), ty = threadIdx.x >> log2_of(lanes), rows = blockDim.x >> log2_of(lanes);
    const int64_t tiles = (a.B + lanes * V - 1) / (lanes * V);
    float *dw = a.dw ? a.dw + blockIdx.x * a.H : nullptr;
    float *db = a.db ? a.db + blockIdx.x * a.H : nullptr;
    float sw[kHeld], sb[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) sw[i] = sb[i] = 0.0f;
    // over the lanes that share a feature's tokens; whole waves come here
    auto across = [&](float s) {
        for (int d = 1; d < lanes; d <<= 1) s += __shfl_xor(s, d, kWave);
        return s;
    };
    float w[kHeld];
    if constexpr (N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t h = ty + int64_t(i) * rows < a.H ? ty + int64_t(i) * rows : 0;
            w[i] = a.w ? weight_at<T>(a, a.w, h) : 1.0f;
        }
    }
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int skip;
        const int64_t b = back_from_end<V>((tile_of(tile, tiles) * lanes + tx) * V, a.B, skip);
        Tile<T, V, N> x, dy;
        x.open(a.x.p, b, a.H, a.x.feature, ty, rows);
        dy.open(a.dy.p, b, a.H, a.dy.feature, ty, rows);
        float mean[V], rstd[V], s[2 * V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            mean[j] = a.mean[b + j];
            rstd[j] = a.rstd[b + j];
            s[j] = s[V + j] = 0.0f;
        }
        x.each([&](int i, int64_t h, const Loaded<T, V> &v) {
            const Loaded<T, V> g = N ? dy.held[i] : dy.get(h);
            if constexpr (!N) w[i] = a.w ? weight_at<T>(a, a.w, h) : 1.0f;
            float fw = 0.0f, fb = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (v[j] - mean[j]) * rstd[j], c = g[j] * w[i];
                s[j] += c;
                s[V + j] = fmaf(c, xh, s[V + j]);
                fw = j >= skip ? fmaf(g[j], xh, fw) : fw;
                fb = j >= skip ? fb + g[j] : fb;
            }
            if constexpr (N) {
                sw[i] += fw;
                sb[i] += fb;
            } else {
                // the lanes of a feature are all here, or none
                fw = across(fw);
                fb = across(fb);
                if (tx == 0) {
                    const bool first = tile == blockIdx.x;
                    if (dw) dw[h] = first ? fw : dw[h] + fw;
                    if (db) db[h] = first ? fb : db[h] + fb;
                }
            }
        });
        if (!a.y.p) continue;
        tile_sum(s, lanes, room);
        x.forget();
        dy.forget();
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) s[j] /= float(a.H);
        x.each([&](int i, int64_t h, const Loaded<T, V> &v) {
            const Loaded<T, V> g = N ? dy.held[i] : dy.get(h);
            if constexpr (!N) w[i] = a.w ? weight_at<T>(a, a.w, h) : 1.0f;
            float out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (v[j] - mean[j]) * rstd[j];
                out[j] = rstd[j] * (g[j] * w[i] - s[j] - xh * s[V + j]);
            }
            store_own<T, V>(out_row<T, V, N>(a.y, i, h, ty, rows, b), skip, out);
        });
    }
    if constexpr (N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float w = across(sw[i]), c = across(sb[i]);
            const int64_t h = ty + int64_t(i) * rows;
            if (tx != 0 || h >= a.H) continue;
            if (dw) dw[h] = w;
            if (db) db[h] = c;
        }
    }
}

// ---- feature-major, many features of few tokens: the features cut too ------------------
//
// Where whole columns fit a workgroup only in tiles of a vector or two, 16 bytes of every cache
// line, the features are cut into chunks: a first launch sums a chunk of kSplitTokens tokens (the
// columns' two sums into `parts`, dw and db into partial rows of the token tile), a second one
// adds the columns' sums and writes dx, reading x and dy again (from a cache, mostly).

constexpr int kSplitTokens = 64, kSplitThreads = 256;

struct SplitArgs {
    Args n;                             // n.dw, n.db: partial sums [tiles][H]
    float *parts;                       // [chunks][2][B]
    int tiles, chunk;                   // chunk: features, a multiple of the rows of a workgroup
};

// f(round, feature, x, dy) for the thread's vectors of its chunk, kAtOnce loads of each together.
template <typename T, int V, typename F>
__device__ __forceinline__ void each_of_chunk(const SplitArgs &a, int64_t first, int ty, int64_t b, F &&f) {
    constexpr int kRows = kSplitThreads / (kSplitTokens / V), kAtOnce = V > 4 ? 2 : 4;
    const T *x = static_cast<const T *>(a.n.x.p) + b, *dy = static_cast<const T *>(a.n.dy.p) + b;
    for (int r0 = 0; r0 < a.chunk; r0 += kRows * kAtOnce) {
        Loaded<T, V> v[kAtOnce], g[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            int64_t h = first + r0 + q * kRows + ty;
            if (h >= a.n.H) h = a.n.H - 1;
            v[q] = load_vec<T, V>(x + h * a.n.x.feature);
            g[q] = load_vec<T, V>(dy + h * a.n.dy.feature);
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int r = r0 + q * kRows + ty;
            f(r, first + r, r < a.chunk && first + r < a.n.H, v[q], g[q]);
        }
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kSplitThreads) void split_sums_kernel(SplitArgs a) {
    constexpr int kLanes = kSplitTokens / V, kWaves = kSplitThreads / kWave, kMaxChunk = 256;
    __shared__ float sums[2][kWaves][kSplitTokens], params[2][kMaxChunk];
    const int tx = threadIdx.x % kLanes, ty = threadIdx.x / kLanes;
    const int64_t task = tile_of(blockIdx.x, gridDim.x), c = task / a.tiles, tile = task - c * a.tiles;
    int skip;
    const int64_t b = back_from_end<V>(tile * kSplitTokens + tx * V, a.n.B, skip);
    float mean[V], rstd[V], s[2][V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        mean[j] = a.n.mean[b + j];
        rstd[j] = a.n.rstd[b + j];
        s[0][j] = s[1][j] = 0.0f;
    }
    each_of_chunk<T, V>(a, c * a.chunk, ty, b, [&](int r, int64_t h, bool in, const Loaded<T, V> &v, const Loaded<T, V> &g) {
        const float w = in ? a.n.w ? weight_at<T>(a.n, a.n.w, h) : 1.0f : 0.0f;
        float fw = 0.0f, fb = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (v[j] - mean[j]) * rstd[j], t = g[j] * w;
            s[0][j] = in ? s[0][j] + t : s[0][j];
            s[1][j] = in ? fmaf(t, xh, s[1][j]) : s[1][j];
            fw = j >= skip ? fmaf(g[j], xh, fw) : fw;
            fb = j >= skip ? fb + g[j] : fb;
        }
        fw = group_reduce<kLanes, AddOp>(fw);
        fb = group_reduce<kLanes, AddOp>(fb);
        if (tx == 0 && in) {
            params[0][r] = fw;
            params[1][r] = fb;
        }
    });
    // over the lanes and waves that have the same tokens
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float t = kLanes == 16 ? sum_rows(s[k][j]) : sum_equal_lanes(s[k][j], kLanes);
            if (lane_id() < kLanes) sums[k][wave_id()][tx * V + j] = t;
        }
    __syncthreads();
    const int i = threadIdx.x % kSplitTokens, k = threadIdx.x / kSplitTokens;
    if (k < 2) {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) t += sums[k][w][i];
        // where lane i / V has its tokens
        const int64_t own = tile * kSplitTokens + i / V * V, at = (own > a.n.B - V ? a.n.B - V : own) + i % V;
        if (at >= own) a.parts[(c * 2 + k) * a.n.B + at] = t;
    }
    const int64_t h = c * a.chunk + threadIdx.x;
    if (int(threadIdx.x) < a.chunk && h < a.n.H) {
        if (a.n.dw) a.n.dw[tile * a.n.H + h] = params[0][threadIdx.x];
        if (a.n.db) a.n.db[tile * a.n.H + h] = params[1][threadIdx.x];
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kSplitThreads) void split_dx_kernel(SplitArgs a, int chunks) {
    constexpr int kLanes = kSplitTokens / V, kWaves = kSplitThreads / kWave;
    __shared__ float sums[2][kWaves][kSplitTokens];
    const int tx = threadIdx.x % kLanes, ty = threadIdx.x / kLanes;
    const int64_t task = tile_of(blockIdx.x, gridDim.x), c = task / a.tiles, tile = task - c * a.tiles;
    {
        const int64_t token = tile * kSplitTokens + lane_id(), at = token < a.n.B ? token : a.n.B - 1;
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll 4
        for (int k = wave_id(); k < chunks; k += kWaves) {
            s0 += a.parts[int64_t(k) * 2 * a.n.B + at];
            s1 += a.parts[(int64_t(k) * 2 + 1) * a.n.B + at];
        }
        sums[0][wave_id()][lane_id()] = s0;
        sums[1][wave_id()][lane_id()] = s1;
    }
    int skip;
    const int64_t b = back_from_end<V>(tile * kSplitTokens + tx * V, a.n.B, skip);
    float mean[V], rstd[V], m0[V], m1[V];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        mean[j] = a.n.mean[b + j];
        rstd[j] = a.n.rstd[b + j];
        // what the lane leaves out may lie before the tile
        const int64_t token = b + j - tile * kSplitTokens;
        const int i = token < 0 ? 0 : int(token);
        m0[j] = m1[j] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            m0[j] += sums[0][w][i];
            m1[j] += sums[1][w][i];
        }
        m0[j] /= float(a.n.H);
        m1[j] /= float(a.n.H);
    }
    T *dx = static_cast<T *>(a.n.y.p) + b;
    each_of_chunk<T, V>(a, c * a.chunk, ty, b, [&](int, int64_t h, bool in, const Loaded<T, V> &v, const Loaded<T, V> &g) {
        if (!in) return;
        const float w = a.n.w ? weight_at<T>(a.n, a.n.w, h) : 1.0f;
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (v[j] - mean[j]) * rstd[j];
            out[j] = rstd[j] * (g[j] * w - m0[j] - xh * m1[j]);
        }
        store_own<T, V>(dx + h * a.n.y.feature, skip, out);
    });
}

// ---- the partial sums of dw and db -----------------------------------------------------

constexpr int kSumFeatures = 32, kSumSlices = 32;    // a cache line a row

__global__ __launch_bounds__(kSumFeatures * kSumSlices) void sum_partials_kernel(
    const float *__restrict__ dw_parts, const float *__restrict__ db_parts, int64_t first, int64_t H,
    int blocks, float *__restrict__ dw, float *__restrict__ db) {
    constexpr int kSumWaves = kSumFeatures * kSumSlices / kWave, kAtOnce = 4;
    __shared__ float s[2][kSumWaves][kSumFeatures];
    const int f = threadIdx.x % kSumFeatures, slice = threadIdx.x / kSumFeatures;
    const int64_t h = first + int64_t(blockIdx.x) * kSumFeatures + f, at = h < H ? h : H - 1;
    float w = 0.0f, b = 0.0f;
    for (int k = slice; k < blocks; k += kSumSlices * kAtOnce) {
        float x[kAtOnce], y[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int row = k + q * kSumSlices, in = row < blocks ? row : blocks - 1;
            x[q] = dw ? dw_parts[in * H + at] : 0.0f;
            y[q] = db ? db_parts[in * H + at] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const bool live = k + q * kSumSlices < blocks;
            w += live ? x[q] : 0.0f;
            b += live ? y[q] : 0.0f;
        }
    }
    // the wave's two slices, then the waves
    w += __shfl_xor(w, kSumFeatures, kWave);
    b += __shfl_xor(b, kSumFeatures, kWave);
    const int wave = threadIdx.x / kWave, lane = lane_id();
    if (lane < kSumFeatures) {
        s[0][wave][lane] = w;
        s[1][wave][lane] = b;
    }
    __syncthreads();
    if (threadIdx.x >= kSumFeatures || h >= H) return;
    w = b = 0.0f;
#pragma unroll
    for (int k = 0; k < kSumWaves; ++k) {
        w += s[0][k][f];
        b += s[1][k][f];
    }
    if (dw) dw[h] = w;
    if (db) db[h] = b;
}

// Rows of partial sums, at most: token-major a workgroup a CU, feature-major as many as tiles.
constexpr int kMaxRowBlocks = 256, kMaxTileBlocks = 512;

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Features of a thread up to which a wave takes a row of the gradient by itself.
constexpr int kTeamFeatures = 16;

// A token-major call: threads that hold a row, N vectors each (0: the row is too long); one wave
// where it needs at most one_wave vectors a lane.
struct RowShape {
    int threads, n;
};

RowShape row_shape(int64_t H, int vec, int most, int one_wave, bool gradient = false) {
    if (H < vec) return {kWave, 1};                  // an element a thread
    const int64_t vectors = up(H, vec);
    if (vectors <= kWave * one_wave) return {kWave, int(up(vectors, kWave))};
    for (int threads = 256; threads <= most; threads *= 2)
        for (int n = 1; n <= 4; ++n)
            if (up(up(vectors, n), kWave) * kWave <= threads && (!gradient || threads <= row_threads(vec, n)))
                return {int(up(up(vectors, n), kWave) * kWave), n};
    return {gradient ? kGradThreads : most, 0};
}

template <typename F> hipError_t with_row(const RowShape &r, F &&f) {
    switch (r.n) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 3: return f(std::integral_constant<int, 3>{});
        case 4: return f(std::integral_constant<int, 4>{});
        default: return f(std::integral_constant<int, 0>{});
    }
}

// A feature-major call: a tile of `lanes` vectors of tokens, the widest that leaves
// about a workgroup a CU, whose threads hold N features each.
struct TileShape {
    int lanes, threads, n, vec;
};

// (In one graph, 200 tiles at least, 128 and 384: forward 1500 x 4096 fp32 12.5, 14.8 and 14.6 us, 4096
// x 4096 bf16 23.4, 28.0 and 32.0, 1024 x 2048 fp32 7.9, 7.2 and 10.1; gradients of the last 12.5,
// 12.3 and 18.4.)
TileShape tile_shape(int64_t H, int64_t B, int64_t stride, int vec, int threads, int most) {
    constexpr int kTiles = 200;
    TileShape t;
    t.vec = B < vec ? 1 : vec;
    t.lanes = kMaxLanes;
    while (t.lanes > 1 && up(B, int64_t(t.lanes) * t.vec) < kTiles) t.lanes /= 2;
    // narrower where registers hold that: 4096 x 4096 fp32 43 -> 27 us, 9216 x 2047 77 -> 67
    const int64_t held = int64_t(threads) * most;
    while (t.lanes > 1 && H <= held && H * t.lanes > held) t.lanes /= 2;
    const int64_t want = H * t.lanes;
    t.threads = threads;
    t.n = 2;
    while (t.n <= most && want > int64_t(threads) * t.n) t.n *= 2;
    // a thread's vectors lie within 32 bits of bytes of their round's first
    if (t.n > most || (int64_t(threads) * stride + B) * 4 >= int64_t(1) << 32) t.n = 0;
    return t;
}

template <int MOST, typename F> hipError_t with_tile(const TileShape &t, F &&f) {
    if constexpr (MOST >= 16) if (t.n == 16) return f(std::integral_constant<int, 16>{});
    switch (t.n) {
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 8: return f(std::integral_constant<int, 8>{});
        default: return f(std::integral_constant<int, 0>{});
    }
}

// One launch per 2^20 workgroups (a launch has below 2^32 threads).
template <typename F> hipError_t over_grid(Args a, int64_t n, F &&launch) {
    constexpr int64_t kMost = 1 << 20;
    for (a.first = 0; a.first < n; a.first += kMost) {
        launch(a, dim3(unsigned(n - a.first < kMost ? n - a.first : kMost)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// A feature-major gradient whose features are cut: 9216 x 64 fp32 35 -> 13 us, 9216 x 700 66 ->
// 31 (bf16 78 -> 22), 4096 x 700 23 -> 16; from here on no size measured is slower by more than a
// twentieth, below (1024 x 700 fp32 11.8 -> 12.5) the third launch costs more.  The workspace, 8
// bytes a feature and token of up to 512, holds the parts (chunks of 64 features at least) and a
// partial row per 64 tokens.
bool is_split(int64_t H, int64_t B, int vec) {
    const bool fits = up(H, 256) * up(B, kSplitTokens) < 1 << 24;    // a launch has below 2^32 threads
    return fits && B >= 8 && B <= 8192 && (H > 2048 || (vec > 4 && H > 1024 && B >= 128));
}

// A launch per 2^26 features (it has below 2^32 threads).
hipError_t launch_sum_partials(const float *dw_parts, const float *db_parts, int64_t H, int blocks, float *dw,
                               float *db, hipStream_t s) {
    constexpr int64_t kMost = int64_t(1) << 26;
    for (int64_t first = 0; first < H; first += kMost) {
        const int64_t n = H - first < kMost ? H - first : kMost;
        hipLaunchKernelGGL(sum_partials_kernel, dim3(unsigned(up(n, kSumFeatures))), dim3(kSumFeatures * kSumSlices),
                           0, s, dw_parts, db_parts, first, H, blocks, dw, db);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t layer_norm_workspace_bytes(int64_t H, int64_t B) {
    const int64_t blocks = B < kMaxTileBlocks ? B : kMaxTileBlocks;
    return 2 * padded(blocks * H * 4);
}

hipError_t launch_layer_norm(int xdtype, int wdtype, int64_t H, int64_t B, bool rows,
                             const void *x, int64_t x_feature, int64_t x_token, const void *weight,
                             const void *bias, float eps, void *y, int64_t y_feature,
                             int64_t y_token, float *mean, float *rstd, hipStream_t s) {
    const Args a{{const_cast<void *>(x), x_feature, x_token}, {y, y_feature, y_token}, {}, weight,
                 bias, wdtype == DARB_F32, H, B, eps, mean, rstd, nullptr, nullptr, 0};
    return with_type(xdtype, [&](auto type) {
        using T = decltype(type);
        if (rows) {
            const RowShape r = row_shape(H, kVec<T>, kMaxThreads, 1);
            return with_row(r, [&](auto n) {
                return over_grid(a, B, [&](const Args &part, dim3 grid) {
                    if (H < kVec<T>)
                        hipLaunchKernelGGL((norm_rows_kernel<T, 1, 1>), grid, dim3(r.threads), 0, s, part);
                    else
                        hipLaunchKernelGGL((norm_rows_kernel<T, kVec<T>, decltype(n)::value>), grid,
                                           dim3(r.threads), 0, s, part);
                });
            });
        }
        const TileShape t = tile_shape(H, B, x_feature > y_feature ? x_feature : y_feature, kVec<T>, kMaxThreads, 16);
        return with_tile<16>(t, [&](auto n) {
            return over_grid(a, up(B, int64_t(t.lanes) * t.vec), [&](const Args &part, dim3 grid) {
                if (t.vec == 1)
                    hipLaunchKernelGGL((norm_columns_kernel<T, 1, decltype(n)::value>), grid,
                                       dim3(t.threads), 0, s, part, t.lanes);
                else
                    hipLaunchKernelGGL((norm_columns_kernel<T, kVec<T>, decltype(n)::value>), grid,
                                       dim3(t.threads), 0, s, part, t.lanes);
            });
        });
    });
}

hipError_t launch_layer_norm_grad(int xdtype, int wdtype, int64_t H, int64_t B, bool rows,
                                  const void *dy, int64_t dy_feature, int64_t dy_token, const void *x,
                                  int64_t x_feature, int64_t x_token, const float *mean,
                                  const float *rstd, const void *weight, void *dx,
                                  int64_t dx_feature, int64_t dx_token, float *dweight,
                                  float *dbias, void *workspace, hipStream_t s) {
    Args a{{const_cast<void *>(x), x_feature, x_token}, {dx, dx_feature, dx_token},
           {const_cast<void *>(dy), dy_feature, dy_token}, weight, nullptr, wdtype == DARB_F32,
           H, B, 0.0f, const_cast<float *>(mean), const_cast<float *>(rstd), nullptr, nullptr, 0};
    return with_type(xdtype, [&](auto type) {
        using T = decltype(type);
        int64_t stride = x_feature > dy_feature ? x_feature : dy_feature;
        if (dx && dx_feature > stride) stride = dx_feature;
        const TileShape t = tile_shape(H, B, stride, kVec<T>, kTileThreads<T>, kMostHeld<T>);
        const RowShape r = row_shape(H, kVec<T>, kMaxThreads, kTeamFeatures / kVec<T>, true);
        const bool waves = r.threads == kWave;
        // Teams of a workgroup: of one wave each, or up to four of 256 threads at most where each
        // has two rows or more.  (Two of 512, or rows that then spill, are slower by a tenth or more.)
        int teams = waves ? kGradThreads / kWave : 1;
        if (!waves && r.threads <= 256 && row_threads(kVec<T>, r.n) == kMaxThreads)
            while (teams < 4 && B >= int64_t(2 * kMaxRowBlocks) * (teams + 1)) ++teams;
        const int64_t tasks = rows ? up(B, teams) : up(B, int64_t(t.lanes) * t.vec);
        const int most = rows && !waves ? kMaxRowBlocks : kMaxTileBlocks;
        const int blocks = tasks < most ? int(tasks) : most;
        if (dweight) a.dw = static_cast<float *>(workspace);
        if (dbias) a.db = reinterpret_cast<float *>(static_cast<char *>(workspace) + padded(blocks * H * 4));
        hipError_t e;
        if (!rows && is_split(H, B, kVec<T>)) {
            SplitArgs p{a, nullptr, int(up(B, kSplitTokens)), 256};
            while (p.chunk > 64 && up(H, p.chunk) * p.tiles < 512) p.chunk /= 2;
            const int64_t chunks = up(H, p.chunk);
            float *next = static_cast<float *>(workspace);
            p.parts = next;
            next += padded(chunks * 2 * B * 4) / 4;
            p.n.dw = dweight ? next : nullptr;
            next += padded(p.tiles * H * 4) / 4;
            p.n.db = dbias ? next : nullptr;
            const dim3 grid{unsigned(chunks * p.tiles)};
            hipLaunchKernelGGL((split_sums_kernel<T, kVec<T>>), grid, dim3(kSplitThreads), 0, s, p);
            e = hipGetLastError();
            if (e == hipSuccess && dx) {
                hipLaunchKernelGGL((split_dx_kernel<T, kVec<T>>), grid, dim3(kSplitThreads), 0, s, p, int(chunks));
                e = hipGetLastError();
            }
            if (e != hipSuccess || (!dweight && !dbias)) return e;
            return launch_sum_partials(p.n.dw, p.n.db, H, p.tiles, dweight, dbias, s);
        }
        if (rows) {
            const dim3 grid{unsigned(blocks)}, threads{unsigned(r.threads * teams)};
            e = with_row(r, [&](auto n) {
                constexpr int N = decltype(n)::value, VT = kVec<T>;
                if (H < VT)
                    hipLaunchKernelGGL((norm_grad_rows_kernel<T, 1, 1, true>), grid, threads, 0, s, a, r.threads);
                else if (waves && N > 0 && N * VT <= kTeamFeatures)
                    hipLaunchKernelGGL((norm_grad_rows_kernel<T, VT, N && N * VT <= kTeamFeatures ? N : 1, true>), grid, threads, 0, s, a, r.threads);
                else
                    hipLaunchKernelGGL((norm_grad_rows_kernel<T, VT, N, false>), grid, threads, 0, s, a, r.threads);
                return hipGetLastError();
            });
        } else {
            e = with_tile<kMostHeld<T>>(t, [&](auto n) {
                if (t.vec == 1)
                    hipLaunchKernelGGL((norm_grad_columns_kernel<T, 1, decltype(n)::value>),
                                       dim3(unsigned(blocks)), dim3(t.threads), 0, s, a, t.lanes);
                else
                    hipLaunchKernelGGL((norm_grad_columns_kernel<T, kVec<T>, decltype(n)::value>),
                                       dim3(unsigned(blocks)), dim3(t.threads), 0, s, a, t.lanes);
                return hipGetLastError();
            });
        }
        if (e != hipSuccess || (!dweight && !dbias)) return e;
        return launch_sum_partials(a.dw, a.db, H, blocks, dweight, dbias, s);
    });
}

}  // namespace darb
