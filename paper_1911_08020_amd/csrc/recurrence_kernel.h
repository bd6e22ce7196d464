// Gated linear recurrence over sequences, and its gradients.
//
//   gate form:    f = sigmoid(z),  h_t = f_t h_{t-1} + (1 - f_t) x_t
//   linear form:  f = z,           h_t = f_t h_{t-1} + x_t
//   gradients:    g_t = dh_t + G_t, G_{t-1} = f_t g_t (G_{T-1} = dh_last, dh_0 = G_{-1}),
//     gate form   dz = (h_{t-1} - x) g f (1 - f),  dx = (1 - f) g
//     linear form dz = h_{t-1} g,                  dx = g
//
// Both are scans of affine maps s -> a s + b (a = f; b = what h_t takes from x_t, or f_t dh_t),
// forwards or backwards in time, and maps compose: (a, b) after (a', b') is (a a', a b' + b).  A
// restart is a map that does not read s at all, carried as a bit beside (a, b): a = 0 would let
// an infinity or NaN of the sequence before through.
//
// Element (o, t, i) lies at o * so + t * st + i: features x columns with the columns contiguous
// has a feature per o and a sequence per i, with the features contiguous the reverse.  A thread
// takes V series that lie side by side over C steps, whose maps it holds in registers from one read
// (V C = 16 forward, 8 for the gradients, which hold four values an element; at twice that registers
// spill: 15.6 -> 16.9 us and 35.5 -> 45.6 in the case below); the workgroup's 256 threads are `lanes`
// such groups by 256 / lanes chunks of time.  Chunks are joined by shuffles inside a wave and through
// LDS between waves, and the workgroup goes on to the next steps with the state it has reached.  Few
// series cannot fill the device so: time is then cut into slabs, a first launch writes each slab's
// map and a second one starts each slab from the maps before it (inputs read twice).  Feature-major
// rows of few sequences would be read in short pieces; such rows are staged whole through LDS, or,
// one sequence's, read in vectors along time, a chunk a vector.
//
// Memory-bound: forward 3 arrays, gradients 6 (linear form 5).  Measured on MI355X: 200 steps of 32
// sequences of 1024 fp32 features 16.0 us (4.9 TB/s), gradients 35.8 (4.4 TB/s: a tile's loads are not
// under way while the one before is joined, and registers leave four waves a SIMD); 65536 steps of
// 1024 bf16 features of one sequence, with restarts, 187 us (the inputs read twice 3.6 TB/s: each
// slab's tiles follow one another; 177 with gates off by |z| 2^-24 of themselves); gradients of 1500
// fp16 rows of 2999 steps, linear form, 14.5 us (3.1 TB/s: rows of 1.5 tiles).
#pragma once

#include "darb_internal.h"
#include "exp_of.h"
#include "float_io.h"
#include "wave.h"

#include <type_traits>

namespace darb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kSlabs = 64;              // at most: a thread folds those before its own

struct Operand {
    const void *p;
    int64_t so, st;
};
struct Result {
    void *p;
    int64_t so, st;
};
struct State {                          // fp32 [o, i]
    float *p;
    int64_t so, si;
};

struct Args {
    Operand z, x, h, dh;                // h, dh: gradients only
    Result out, out2;                   // h, or dz and dx
    State in, last;                     // h0 and h_last, or dh_last and dh0
    State h0;                           // gradients: the state before the first step
    const uint8_t *resets;
    int64_t rt, ro, ri;                 // its strides
    int64_t T, W, O;
    int64_t groups;                     // groups of V series
    int lanes;                          // groups of a workgroup, a power of two
    int slabs;
    int64_t slab_steps;
    int64_t first_block;                // of this launch
    float *maps;                        // [2][slabs][series] (a, b); null: one launch
    float *enters;                      // [series] the state before the scan
    uint8_t *cuts;                      // [slabs][series]
};

template <int V, bool CUTS> struct Map {
    float a[V], b[V];
    uint32_t cut;                       // bit v: restarted
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int v = 0; v < V; ++v) a[v] = 1.0f, b[v] = 0.0f;
        cut = 0;
    }
    // this after `m`
    __device__ __forceinline__ void after(const Map &m) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            b[v] = CUTS && (cut >> v) & 1 ? b[v] : a[v] * m.b[v] + b[v];
            a[v] *= m.a[v];
        }
        if (CUTS) cut |= m.cut;
    }
    __device__ __forceinline__ float of(int v, float s) const {
        return CUTS && (cut >> v) & 1 ? b[v] : a[v] * s + b[v];
    }
};

template <int V, bool CUTS> __device__ __forceinline__ Map<V, CUTS> map_up(const Map<V, CUTS> &m, int lanes) {
    Map<V, CUTS> r;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        r.a[v] = __shfl_up(m.a[v], lanes);
        r.b[v] = __shfl_up(m.b[v], lanes);
    }
    r.cut = CUTS ? uint32_t(__shfl_up(int(m.cut), lanes)) : 0;
    return r;
}

// f = sigmoid(z) = 1 / (1 + e^-z) and u = 1 - f, each off by at most 9 2^-24 of itself, however small
// it is (down to 2^-126): u is e^-z f where that is the smaller one.
__device__ __forceinline__ void gates(float z, float &f, float &u) {
    const float e = exp_of(-z);
    f = __builtin_amdgcn_rcpf(1.0f + e);
    u = z < 0.0f ? 1.0f - f : e * f;
}

template <typename T, int V> struct Raw {
    typename VecOf<T, V>::Type v;
    __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const typename VecOf<T, V>::Type *>(p); }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (V == 1) return float(v);
        else return float(v[i]);
    }
};

// LDS place of element i: rows of 32 are moved on by one word, so that chunks that start on
// multiples of 8 spread over the banks.
__device__ __forceinline__ int staged_at(int i) { return i + (i >> 5); }

enum { kDirect, kStaged, kAlong };      // see the top of the file

template <typename T, int V, int C, bool GATE, bool BACK, bool RESETS, int LAYOUT>
__global__ __launch_bounds__(kThreads, 4) void recurrence_kernel(Args k) {
    constexpr bool STAGED = LAYOUT == kStaged, ALONG = LAYOUT == kAlong;
    constexpr int kArrays = BACK ? (GATE ? 4 : 3) : 2;      // staged: z, x; z, dh, h, x
    constexpr int kRoom = STAGED ? kThreads * C + kThreads * C / 32 : 1;
    __shared__ T staged[STAGED ? kArrays : 1][kRoom];
    __shared__ float total[2][kWaves][2][V][kWave];
    __shared__ uint32_t total_cut[2][kWaves][kWave];

    const int lanes = k.lanes, chunks = kThreads / lanes;
    const int tid = int(threadIdx.x), g = tid & (lanes - 1), c = tid / lanes;
    const int lane = tid & (kWave - 1), w = wave_id();
    const int64_t per = k.W / V;                            // groups of an o
    const int64_t blocks = STAGED || ALONG ? k.O : (k.groups + lanes - 1) / lanes;
    const int64_t number = k.first_block + blockIdx.x;
    const int slab = int(number / blocks);
    const int64_t block = number - slab * blocks;
    // threads behind the last group read with it, and write nothing
    const int64_t group = STAGED || ALONG ? 0 : block * lanes + g < k.groups ? block * lanes + g : k.groups - 1;
    const int64_t o = STAGED || ALONG ? block : group / per;
    const int64_t i = STAGED || ALONG ? g : (group - o * per) * V;
    const bool mine = STAGED || ALONG ? g < k.W : block * lanes + g < k.groups;
    // the thread's series at step 0
    auto series_of = [&](const Operand &q) { return static_cast<const T *>(q.p) + o * q.so + i; };
    const bool first_launch = k.maps && !k.out.p;           // only the slabs' maps
    const int64_t t0 = slab * k.slab_steps;
    const int64_t steps = k.T - t0 < k.slab_steps ? k.T - t0 : k.slab_steps;
    const int64_t series = k.O * k.W, at = o * k.W + i;

    // the state that enters the slab, in the direction of the scan
    float state[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        state[v] = mine && k.in.p ? k.in.p[o * k.in.so + (i + v) * k.in.si] : 0.0f;
    if (first_launch && c == 0 && slab == (BACK ? k.slabs - 1 : 0)) {
        // the second launch may write h_last where h0 is
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (mine) k.enters[at + v] = state[v];
    }
    if (k.maps && !first_launch) {
        const int before = BACK ? k.slabs - 1 - slab : slab;
#pragma unroll 4
        for (int q = 0; q < before; ++q) {
            const int64_t from = int64_t(BACK ? k.slabs - 1 - q : q) * series + at;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t e = from + v;
                const float a = k.maps[e], b = k.maps[e + k.slabs * series];
                state[v] = RESETS && k.cuts[e] ? b : a * state[v] + b;
            }
        }
    }
    Map<V, RESETS> all;                                     // first launch: the slab's map
    all.none();

    const int64_t tile = int64_t(chunks) * C;
    // kDirect: where the chunk's first step is (in the direction of the scan), and how far a step takes
    const int64_t begin = BACK ? t0 + steps - 1 - c * C : t0 + c * C, way = BACK ? -1 : 1;
    struct Cursor {
        const T *p;
        int64_t st;
    };
    auto cursor = [&](const Operand &q) { return Cursor{series_of(q) + begin * q.st, q.st * way}; };
    Cursor zc = cursor(k.z), xc = cursor(k.x), hc = cursor(k.h), gc = cursor(k.dh);
    auto writer = [&](const Result &q) { return cursor({q.p, q.so, q.st}); };
    Cursor oc = writer(k.out), oc2 = writer(k.out2);
    // kDirect: z and x (or dh) of a tile of `ts` steps, `ahead` tiles from the cursors; steps that are
    // not there read the tile's last one
    Raw<T, V> rz[C], rb[C];
    auto bring = [&](int ts, int ahead) {
        const Cursor &second = BACK ? gc : xc;
        const T *zp = zc.p + ahead * tile * zc.st, *bp = second.p + ahead * tile * second.st;
        auto all_of = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int64_t d = whole || c * C + j < ts ? j : ts - 1 - c * C;
                rz[j].load(zp + d * zc.st);
                rb[j].load(bp + d * second.st);
            }
        };
        if (ts == tile) all_of(std::true_type{});
        else all_of(std::false_type{});
    };
    auto steps_of = [&](int64_t done) { return int(steps - done < tile ? steps - done : tile); };
    constexpr bool kAhead = LAYOUT == kDirect && !BACK;     // the gradients hold too much for it: 35.5 -> 41 us
    if constexpr (kAhead) bring(steps_of(0), 0);
    int turn = 0;
    for (int64_t done = 0; done < steps; done += tile, turn ^= 1) {
        // Scan position p = done + c * C + j is step t0 + p, or counted from the slab's end.
        const int p0 = c * C;
        const int tsteps = steps_of(done);
        const int64_t ta = BACK ? t0 + steps - done - tsteps : t0 + done;  // the tile's first step
        auto step = [&](int j) {                            // in the tile, kept inside it
            const int p = p0 + j < tsteps ? p0 + j : tsteps - 1;
            return BACK ? tsteps - 1 - p : p;
        };
        const int live = mine ? tsteps - p0 : 0;           // steps j < live are the thread's
        float f[C][V], b[C][V], u[BACK && GATE ? C : 1][V]; // f, what a step adds or dh, 1 - f
        Raw<T, V> y[BACK ? C : 1], xs[BACK && GATE ? C : 1];
        float y0[BACK ? V : 1];                             // the state before the first step
        uint64_t cuts = 0;
        if constexpr (BACK) {
#pragma unroll
            for (int v = 0; v < V; ++v) y0[v] = 0.0f;
        }
        if constexpr (STAGED) {
            // the tile's steps of the row lie together
            const int count = int(tsteps * k.W);
            auto row = [&](const Operand &q) { return static_cast<const T *>(q.p) + o * q.so + ta * k.W; };
            const T *zr = row(k.z), *xr = row(k.x), *hr = row(k.h), *gr = row(k.dh);
            const bool start = BACK && ta == 0;             // h at -1 is h0
            auto bring = [&](T *to, const T *from) {
                for (int e = tid * 4; e < count; e += kThreads * 4) {
                    if (e + 4 <= count) {
                        Raw<T, 4> v;
                        v.load(from + e);
#pragma unroll
                        for (int q = 0; q < 4; ++q) to[staged_at(e + q)] = v.v[q];
                    } else {
                        for (int q = e; q < count; ++q) to[staged_at(q)] = from[q];
                    }
                }
            };
            bring(staged[0], zr);
            bring(staged[1], BACK ? gr : xr);
            if constexpr (BACK) {
                if (!first_launch) {
                    if (start) {
                        for (int e = tid; e < count; e += kThreads) staged[2][staged_at(e)] = e < k.W ? T(0) : hr[e - k.W];
                    } else {
                        bring(staged[2], hr - k.W);
                    }
                    if constexpr (GATE) bring(staged[kArrays - 1], xr);
                }
            }
            __syncthreads();
        }
        if constexpr (ALONG) {
            // the chunk's steps lie side by side: ascending, or backwards from `low` up
            const int64_t low = ta + (BACK ? tsteps - p0 - C : p0);
            auto bring = [&](Raw<T, V> (&to)[C], const T *from, int64_t at) {
                if (live >= C && at >= 0) {
                    const Loaded<T, C> v = load_vec<T, C>(from + at);
#pragma unroll
                    for (int j = 0; j < C; ++j) to[j].v = v.raw[BACK ? C - 1 - j : j];
                } else {
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        const int64_t t = at - low + ta + step(j);
                        to[j].v = j < live && t >= 0 ? from[t] : T(0);
                    }
                }
            };
            bring(rz, series_of(k.z), low);
            bring(rb, series_of(BACK ? k.dh : k.x), low);
            if constexpr (BACK) {
                if (!first_launch) {
                    bring(y, series_of(k.h), low - 1);
                    if constexpr (GATE) bring(xs, series_of(k.x), low);
                }
            }
        } else if constexpr (STAGED) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int s = staged_at(mine ? step(j) * int(k.W) + g : 0);
                rz[j].v = staged[0][s];
                rb[j].v = staged[1][s];
                if constexpr (BACK) {
                    if (!first_launch) {
                        y[j].v = staged[2][s];
                        if constexpr (GATE) xs[j].v = staged[kArrays - 1][s];
                    }
                }
            }
        } else if constexpr (BACK) {
            bring(tsteps, 0);
            if (!first_launch) {
                auto rest = [&](auto whole) {
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        const int64_t d = whole || p0 + j < tsteps ? j : tsteps - 1 - p0;
                        // the state before; step 0's is not in h
                        y[j].load(hc.p + (whole || ta + step(j) > 0 ? d + 1 : d) * hc.st);
                        if constexpr (GATE) xs[j].load(xc.p + d * xc.st);
                    }
                };
                if (tsteps == tile && ta > 0) rest(std::true_type{});
                else rest(std::false_type{});
            }
        }
        if (BACK && !first_launch && k.h0.p && ta == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (mine) y0[v] = k.h0.p[o * k.h0.so + (i + v) * k.h0.si];
        }
        if constexpr (RESETS) {
            const uint8_t *r = k.resets + ta * k.rt + o * k.ro + (mine ? i * k.ri : 0);
            if (V == 1 || k.ri == 0) {                      // one sequence: all its features
                uint8_t first[C];
#pragma unroll
                for (int j = 0; j < C; ++j) first[j] = r[step(j) * k.rt];
#pragma unroll
                for (int j = 0; j < C; ++j) cuts |= first[j] ? uint64_t((1u << V) - 1) << (j * V) : 0;
            } else {
#pragma unroll
                for (int j = 0; j < C; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        cuts |= r[step(j) * k.rt + v] ? uint64_t(1) << (j * V + v) : 0;
            }
        }
        if (RESETS && live < C) cuts &= live > 0 ? (uint64_t(1) << (live * V)) - 1 : 0;   // the steps that are there
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[j][v] = rz[j][v];
                b[j][v] = rb[j][v];
                if constexpr (GATE) {
                    float share;
                    gates(f[j][v], f[j][v], share);
                    if constexpr (BACK) u[j][v] = share;
                    else b[j][v] *= share;
                }
            }
        if constexpr (kAhead) {                             // the next tile's loads beside this one's scan
            if (done + tile < steps) bring(steps_of(done + tile), 1);
        }
        if (tsteps < tile) {                                // steps that are not there change nothing
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (j >= live) {
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] = 1.0f, b[j][v] = 0.0f;
                }
        }
        // the chunk's map; backwards b holds dh, and a step is f (dh + s)
        Map<V, RESETS> m;
        m.none();
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t cut = RESETS ? uint32_t(cuts >> (j * V)) & ((1u << V) - 1) : 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float in = BACK ? f[j][v] * b[j][v] : b[j][v];
                const bool reset = RESETS && (cut >> v) & 1;
                m.b[v] = reset ? (BACK ? 0.0f : in) : f[j][v] * m.b[v] + in;
                m.a[v] *= f[j][v];
            }
            if (RESETS) m.cut |= cut;
        }
        // joined over the wave's chunks, then over the waves
        float enter[V];
        if (chunks == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) enter[v] = state[v], state[v] = m.of(v, state[v]);
            if (first_launch) {
                m.after(all);
                all = m;
            }
        } else {
            for (int d = lanes; d < kWave; d <<= 1) {
                const Map<V, RESETS> up = map_up(m, d);
                if (lane >= d) m.after(up);
            }
            // a wave holds `lanes` groups, or 64 of them
            if (lane >= kWave - lanes) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    total[turn][w][0][v][lane] = m.a[v];
                    total[turn][w][1][v][lane] = m.b[v];
                }
                if (RESETS) total_cut[turn][w][lane] = m.cut;
            }
            Map<V, RESETS> before;
            before.none();
            if (lanes < kWave) {
                const Map<V, RESETS> up = map_up(m, lanes);
                if (lane >= lanes) before = up;
            }
            __syncthreads();
            const int apart = lanes <= kWave ? 1 : lanes / kWave, last = lanes < kWave ? kWave - lanes + g : lane;
            const int from = lanes <= kWave ? 0 : w & (apart - 1);
            for (int q = from; q < kWaves; q += apart) {
                Map<V, RESETS> t;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    t.a[v] = total[turn][q][0][v][last];
                    t.b[v] = total[turn][q][1][v][last];
                }
                t.cut = RESETS ? total_cut[turn][q][last] : 0;
                if (q == w) {
#pragma unroll
                    for (int v = 0; v < V; ++v) enter[v] = before.of(v, state[v]);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) state[v] = t.of(v, state[v]);
                if (first_launch) {
                    t.after(all);
                    all = t;
                }
            }
        }
        if (first_launch) {
            if constexpr (STAGED) __syncthreads();          // the tile is read
            if constexpr (LAYOUT == kDirect) {
                zc.p += tile * zc.st;
                xc.p += tile * xc.st;
                gc.p += tile * gc.st;
            }
            continue;
        }
        // the steps again, from the state that enters the chunk
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (j < live) {
                const int tj = step(j);
                const int64_t t = ta + tj;
                const uint32_t cut = RESETS ? uint32_t(cuts >> (j * V)) & ((1u << V) - 1) : 0;
                float r[V], r2[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const bool reset = RESETS && (cut >> v) & 1;
                    if constexpr (!BACK) {
                        enter[v] = reset ? b[j][v] : f[j][v] * enter[v] + b[j][v];
                        r[v] = enter[v];
                    } else {
                        const float gr = b[j][v] + enter[v];
                        const float past = reset ? 0.0f : t > 0 ? y[j][v] : y0[v];
                        if constexpr (GATE) {
                            r[v] = (past - xs[j][v]) * gr * (f[j][v] * u[j][v]);
                            r2[v] = u[j][v] * gr;
                        } else {
                            r[v] = past * gr;
                            r2[v] = gr;
                        }
                        enter[v] = reset ? 0.0f : f[j][v] * gr;
                    }
                }
                if constexpr (STAGED) {
                    const int s = staged_at(int(tj * k.W) + g);
                    staged[0][s] = T(r[0]);
                    if constexpr (BACK) staged[1][s] = T(r2[0]);
                } else if constexpr (ALONG) {
                    f[j][0] = r[0];
                    if constexpr (BACK) b[j][0] = r2[0];
                } else {
                    store_vec<T, V>(const_cast<T *>(oc.p + j * oc.st), r);
                    if constexpr (BACK) store_vec<T, V>(const_cast<T *>(oc2.p + j * oc2.st), r2);
                }
            }
        }
        if constexpr (ALONG) {
            const int64_t low = ta + (BACK ? tsteps - p0 - C : p0);
            auto put = [&](void *p, int64_t so, float (&from)[C][V]) {
                T *to = static_cast<T *>(p) + o * so;
                if (live >= C) {
                    float v[C];
#pragma unroll
                    for (int j = 0; j < C; ++j) v[BACK ? C - 1 - j : j] = from[j][0];
                    store_vec<T, C>(to + low, v);
                } else {
#pragma unroll
                    for (int j = 0; j < C; ++j)
                        if (j < live) to[ta + step(j)] = T(from[j][0]);
                }
            };
            put(k.out.p, k.out.so, f);
            if constexpr (BACK) put(k.out2.p, k.out2.so, b);
        }
        if constexpr (LAYOUT == kDirect) {
            zc.p += tile * zc.st;
            xc.p += tile * xc.st;
            oc.p += tile * oc.st;
            if constexpr (BACK) {
                hc.p += tile * hc.st;
                gc.p += tile * gc.st;
                oc2.p += tile * oc2.st;
            }
        }
        if constexpr (STAGED) {
            __syncthreads();
            const int count = int(tsteps * k.W);
            T *out = static_cast<T *>(k.out.p) + o * k.out.so + ta * k.W;
            T *out2 = BACK ? static_cast<T *>(k.out2.p) + o * k.out2.so + ta * k.W : nullptr;
            for (int e = tid; e < count; e += kThreads) {
                out[e] = staged[0][staged_at(e)];
                if constexpr (BACK) out2[e] = staged[1][staged_at(e)];
            }
            __syncthreads();
        }
    }
    if (c != 0) return;
    if (first_launch) {
        const int64_t to = int64_t(slab) * series;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (mine) {
                k.maps[to + at + v] = all.a[v];
                k.maps[to + k.slabs * series + at + v] = all.b[v];
                if (RESETS) k.cuts[to + at + v] = uint8_t((all.cut >> v) & 1);
            }
    } else if (k.last.p && slab == (BACK ? 0 : k.slabs - 1)) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (mine) k.last.p[o * k.last.so + (i + v) * k.last.si] = state[v];
    }
}

// How a call is cut: see the top of the file.
struct Cut {
    int layout, vector;
    int lanes, slabs;
    int64_t groups, slab_steps;
};

constexpr int kVector = 2;              // series of a thread, where W is a multiple of it
template <bool BACK> constexpr int kSteps = BACK ? 4 : 8;
constexpr int kRowSteps = 8;

inline Cut cut_of(int V, int C, int size, bool rows, int64_t T, int64_t W, int64_t O) {
    Cut k;
    if (W % V != 0) V = 1;
    // Feature-major rows that would be read in pieces of less than 64 bytes, unless they are short: 200
    // steps of 1024 fp32 features, 8 sequences 7.5 us through LDS and 11.7 directly (gradients 12.3 and
    // 16.2), 16 sequences 11.9 and 9.6 (18.5 and 17.3); 48 steps of 8 sequences 6.3 and 5.5.  Of fp16,
    // 16 sequences 13.6 and 14.6 (20.3 and 17.9: the gradients would rather go directly), 32 sequences
    // 24.1 and 14.1 (36.1 and 20.5).
    k.layout = rows || W * size >= 64 || T < 64 ? kDirect : W == 1 ? kAlong : kStaged;
    if (k.layout != kDirect) {
        V = 1;
        C = kRowSteps;
    }
    // lanes side by side take at least a line of 128 bytes
    int chunks = 1;
    while (chunks < 2 * V * size && int64_t(chunks) * C < T) chunks *= 2;
    k.lanes = kThreads / chunks;
    if (k.layout != kDirect) {
        k.lanes = 1;
        while (k.lanes < W) k.lanes *= 2;
    }
    k.groups = k.layout != kDirect ? O : O * (W / V);
    k.vector = V;
    const int64_t blocks = k.layout != kDirect ? O : (k.groups + k.lanes - 1) / k.lanes;
    const int64_t tile = int64_t(kThreads / k.lanes) * C;
    const int64_t tiles = (T + tile - 1) / tile;
    // Slabs where workgroups are fewer than compute units and have more than a few tiles each, which
    // the second launch and the second reading have to earn: 2048 steps of 1024 fp32 features, one
    // sequence (32 workgroups) 34.4 -> 12.6 us, gradients 67.6 -> 18.8; four 36.1 -> 33.0, 70.8 -> 46.1;
    // eight (256 workgroups) 38.2 -> 59.6, 101 -> 94.5.  256 rows of 4096 steps (two tiles) 6.3 -> 9.2.
    int64_t slabs = blocks < 256 && tiles > 4 ? (1024 + blocks - 1) / blocks : 1;
    if (slabs > kSlabs) slabs = kSlabs;
    if (slabs > tiles) slabs = tiles;
    k.slab_steps = (tiles + slabs - 1) / slabs * tile;
    k.slabs = int((T + k.slab_steps - 1) / k.slab_steps);
    return k;
}

inline int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename T, bool GATE, bool BACK>
hipError_t launch(const RecurrenceCall &c, hipStream_t s) {
    constexpr int V = kVector, C = kSteps<BACK>;
    const int64_t W = c.rows ? c.H : c.batch, O = c.rows ? c.batch : c.H;
    const Cut cut = cut_of(V, C, int(sizeof(T)), c.rows, c.T, W, O);
    auto stride = [&](const RecurrenceMatrix &m, int64_t &so, int64_t &st) {
        so = c.rows ? m.batch : m.feature;
        st = (c.rows ? m.batch : 1) * c.batch;
    };
    Args k{};
    k.z.p = c.gate.p;
    k.x.p = c.x.p;
    k.h.p = c.h.p;
    k.dh.p = c.dh.p;
    stride(c.gate, k.z.so, k.z.st);
    stride(c.x, k.x.so, k.x.st);
    stride(c.h, k.h.so, k.h.st);
    stride(c.dh, k.dh.so, k.dh.st);
    stride(c.out, k.out.so, k.out.st);
    stride(c.out2, k.out2.so, k.out2.st);
    auto state = [&](const RecurrenceMatrix &m) {
        return State{static_cast<float *>(m.p), c.rows ? m.batch : m.feature, c.rows ? m.feature : m.batch};
    };
    k.in = state(c.in);
    k.last = state(c.last);
    k.h0 = state(c.h0);
    k.resets = c.resets;
    k.rt = c.batch;
    k.ro = c.rows ? 1 : 0;
    k.ri = c.rows ? 0 : 1;
    k.T = c.T;
    k.W = W;
    k.O = O;
    k.groups = cut.groups;
    k.lanes = cut.lanes;
    k.slabs = cut.slabs;
    k.slab_steps = cut.slab_steps;
    const int64_t blocks = cut.layout != kDirect ? O : (cut.groups + cut.lanes - 1) / cut.lanes;
    auto go = [&](const Args &a) {
        return over_blocks(blocks * cut.slabs, kThreads, [&](int64_t first, unsigned n) {
            Args b = a;
            b.first_block = first;
            auto run = [&](auto resets) {
                constexpr bool kResets = decltype(resets)::value;
                auto kernel = recurrence_kernel<T, V, C, GATE, BACK, kResets, kDirect>;
                if (cut.layout == kStaged) kernel = recurrence_kernel<T, 1, kRowSteps, GATE, BACK, kResets, kStaged>;
                else if (cut.layout == kAlong) kernel = recurrence_kernel<T, 1, kRowSteps, GATE, BACK, kResets, kAlong>;
                else if (cut.vector == 1) kernel = recurrence_kernel<T, 1, C, GATE, BACK, kResets, kDirect>;
                hipLaunchKernelGGL(kernel, dim3(n), dim3(kThreads), 0, s, b);
            };
            if (c.resets) run(std::true_type{});
            else run(std::false_type{});
        });
    };
    if (cut.slabs > 1) {
        const int64_t series = W * O;
        k.maps = static_cast<float *>(c.workspace);
        k.enters = k.maps + padded(8 * series * cut.slabs) / 4;
        k.cuts = reinterpret_cast<uint8_t *>(k.enters) + padded(4 * series);
        const hipError_t e = go(k);
        if (e != hipSuccess) return e;
        k.in = {k.enters, W, 1};
    }
    k.out.p = c.out.p;
    k.out2.p = c.out2.p;
    return go(k);
}

// A call of type T, in the source file of that type.
template <typename T> hipError_t launch_type(const RecurrenceCall &c, hipStream_t s) {
    const bool gate = c.form == DARB_RECURRENCE_GATE;
    if (c.back) return gate ? launch<T, true, true>(c, s) : launch<T, false, true>(c, s);
    return gate ? launch<T, true, false>(c, s) : launch<T, false, false>(c, s);
}

}  // namespace
}  // namespace darb
