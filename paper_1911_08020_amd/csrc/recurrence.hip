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
// takes kV series that lie side by side over kSteps steps, whose maps it holds in registers from
// one read; the workgroup's 256 threads are `lanes` such groups by 256 / lanes chunks of time.
// Chunks are joined by shuffles inside a wave and through LDS between waves, and the workgroup
// goes on to the next steps with the state it has reached.  Few series cannot fill the device so:
// time is then cut into slabs, a first launch writes each slab's map and a second one starts each
// slab from the maps before it (inputs read twice).  Feature-major rows of few sequences would
// be read in short pieces; such rows are staged whole through LDS.
//
// Memory-bound: forward 3 arrays, gradients 6 (5).
#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

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
    int64_t groups;                     // groups of kV series
    int lanes;                          // groups of a workgroup, a power of two
    int slabs;
    int64_t slab_steps;
    int64_t first_block;                // of this launch
    float *maps;                        // [2][slabs][series] (a, b); null: one launch
    float *enters;                      // [series] the state before the scan
    uint8_t *cuts;                      // [slabs][series]
};

template <int V> struct Map {
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
            b[v] = (cut >> v) & 1 ? b[v] : a[v] * m.b[v] + b[v];
            a[v] *= m.a[v];
        }
        cut |= m.cut;
    }
    __device__ __forceinline__ float of(int v, float s) const {
        return (cut >> v) & 1 ? b[v] : a[v] * s + b[v];
    }
};

template <int V> __device__ __forceinline__ Map<V> map_up(const Map<V> &m, int lanes) {
    Map<V> r;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        r.a[v] = __shfl_up(m.a[v], lanes);
        r.b[v] = __shfl_up(m.b[v], lanes);
    }
    r.cut = uint32_t(__shfl_up(int(m.cut), lanes));
    return r;
}

// sigmoid(z) and 1 - sigmoid(z), each to a few units in its last place: the smaller of the two is
// s = e^-|z| / (1 + e^-|z|), kept with the sign bit set where it is 1 - sigmoid(z); the other is
// 1 - s.
__device__ __forceinline__ float gate_share(float z) {
    const float e = expf(-fabsf(z));
    const float s = e * __builtin_amdgcn_rcpf(1.0f + e);
    return z >= 0.0f ? -s : s;          // a NaN stays one
}
__device__ __forceinline__ float gate_f(float s) { return __float_as_int(s) < 0 ? 1.0f + s : s; }
__device__ __forceinline__ float gate_u(float s) { return __float_as_int(s) < 0 ? -s : 1.0f - s; }

// V elements, or the first n of them (a whole vector where ALL: the address of the others is
// valid too).
template <typename T, int V> struct Raw {
    typename VecOf<T, V>::Type v;
    __device__ __forceinline__ void load(const T *p, int n, bool whole) {
        if (whole) {
            v = *reinterpret_cast<const typename VecOf<T, V>::Type *>(p);
        } else if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < n ? p[i] : T(0);
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (V == 1) return float(v);
        else return float(v[i]);
    }
};

template <typename T, int V> __device__ __forceinline__ void store_n(T *p, int n, const float (&f)[V]) {
    if (n == V) {
        store_vec<T, V>(p, f);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < n) p[v] = T(f[v]);
    }
}

// LDS place of element i: rows of 32 are moved on by one word, so that chunks that start on
// multiples of 8 spread over the banks.
__device__ __forceinline__ int staged_at(int i) { return i + (i >> 5); }

template <typename T, int V, int C, bool GATE, bool BACK, bool STAGED>
__global__ __launch_bounds__(kThreads) void recurrence_kernel(Args k) {
    constexpr int kArrays = BACK ? (GATE ? 4 : 3) : 2;      // staged: z, x; z, dh, h, x
    constexpr int kRoom = STAGED ? kThreads * C + kThreads * C / 32 : 1;
    __shared__ T staged[STAGED ? kArrays : 1][kRoom];
    __shared__ float total[2][kWaves][2][V][kWave];
    __shared__ uint32_t total_cut[2][kWaves][kWave];

    const int lanes = k.lanes, chunks = kThreads / lanes;
    const int tid = int(threadIdx.x), g = tid & (lanes - 1), c = tid / lanes;
    const int lane = tid & (kWave - 1), w = wave_id();
    const int64_t per = (k.W + V - 1) / V;                  // groups of an o
    const int64_t blocks = STAGED ? k.O : (k.groups + lanes - 1) / lanes;
    const int64_t number = k.first_block + blockIdx.x;
    const int slab = int(number / blocks);
    const int64_t block = number - slab * blocks;
    const int64_t group = STAGED ? 0 : block * lanes + g;
    const int64_t o = STAGED ? block : group / per;
    const int64_t i = STAGED ? g : (group - o * per) * V;
    // the series of this thread: none, some or all of V
    const int64_t left = STAGED ? k.W - g : group < k.groups ? k.W - i : 0;
    const int n = left <= 0 ? 0 : left < V ? int(left) : V;

    // A thread without series reads those of the first group, whole, and writes nothing; where a
    // wave has a group that is not whole, all its loads go element by element.
    const bool whole = k.W >= V && __ballot(n != V && n != 0) == 0;
    const int64_t lo = n ? o : 0, li = n ? i : 0;
    const T *z = static_cast<const T *>(k.z.p) + lo * k.z.so + li;
    const T *x = static_cast<const T *>(k.x.p) + lo * k.x.so + li;
    const T *h = BACK ? static_cast<const T *>(k.h.p) + lo * k.h.so + li : nullptr;
    const T *dh = BACK ? static_cast<const T *>(k.dh.p) + lo * k.dh.so + li : nullptr;
    const bool first_launch = k.maps && !k.out.p;           // only the slabs' maps
    const int64_t t0 = slab * k.slab_steps;
    const int64_t steps = k.T - t0 < k.slab_steps ? k.T - t0 : k.slab_steps;
    const int64_t series = k.O * k.W, at = o * k.W + i;

    // the state that enters the slab, in the direction of the scan
    float state[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        state[v] = v < n && k.in.p ? k.in.p[o * k.in.so + (i + v) * k.in.si] : 0.0f;
    if (first_launch && c == 0 && slab == (BACK ? k.slabs - 1 : 0)) {
        // the second launch may write h_last where h0 is
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < n) k.enters[at + v] = state[v];
    }
    if (k.maps && !first_launch) {
        const int before = BACK ? k.slabs - 1 - slab : slab;
#pragma unroll 4
        for (int q = 0; q < before; ++q) {
            const int64_t from = int64_t(BACK ? k.slabs - 1 - q : q) * series + (n ? at : 0);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t e = from + (v < n ? v : 0);
                const float a = k.maps[e], b = k.maps[e + k.slabs * series];
                state[v] = k.cuts[e] ? b : a * state[v] + b;
            }
        }
    }
    Map<V> all;                                             // first launch: the slab's map
    all.none();

    const int64_t tile = int64_t(chunks) * C;
    int turn = 0;
    for (int64_t done = 0; done < steps; done += tile, turn ^= 1) {
        // Scan position p = done + c * C + j is step t0 + p, or counted from the slab's end.
        const int p0 = c * C;
        const int tsteps = int(steps - done < tile ? steps - done : tile);
        const int64_t ta = BACK ? t0 + steps - done - tsteps : t0 + done;  // the tile's first step
        auto step = [&](int j) {                            // in the tile, kept inside it
            const int p = p0 + j < tsteps ? p0 + j : tsteps - 1;
            return BACK ? tsteps - 1 - p : p;
        };
        const int live = n > 0 ? tsteps - p0 : 0;           // steps j < live are the thread's
        float f[C][V], b[C][V];                             // f (its share, for both uses) and b
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
            for (int e = tid; e < count; e += kThreads) {
                const int s = staged_at(e);
                staged[0][s] = zr[e];
                if constexpr (!BACK) {
                    staged[1][s] = xr[e];
                } else {
                    staged[1][s] = gr[e];
                    if (!first_launch) {
                        staged[2][s] = start && e < k.W ? T(0) : hr[e - k.W];
                        if constexpr (GATE) staged[kArrays - 1][s] = xr[e];
                    }
                }
            }
            __syncthreads();
        }
        Raw<T, V> rz[C], rb[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int tj = step(j);
            const int64_t t = ta + tj;
            if constexpr (STAGED) {
                if constexpr (V == 1) {
                    const int s = staged_at(n ? int(tj * k.W) + g : 0);
                    rz[j].v = staged[0][s];
                    rb[j].v = staged[1][s];
                    if constexpr (BACK) {
                        if (!first_launch) {
                            y[j].v = staged[2][s];
                            if constexpr (GATE) xs[j].v = staged[kArrays - 1][s];
                        }
                    }
                }
            } else {
                rz[j].load(z + t * k.z.st, n, whole);
                if constexpr (!BACK) {
                    rb[j].load(x + t * k.x.st, n, whole);
                } else {
                    rb[j].load(dh + t * k.dh.st, n, whole);
                    if (!first_launch) {
                        y[j].load(h + (t > 0 ? t - 1 : 0) * k.h.st, n, whole);
                        if constexpr (GATE) xs[j].load(x + t * k.x.st, n, whole);
                    }
                }
            }
        }
        if (BACK && !first_launch && k.h0.p && ta == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v < n) y0[v] = k.h0.p[o * k.h0.so + (i + v) * k.h0.si];
        }
        if (k.resets) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const uint8_t *r = k.resets + (ta + step(j)) * k.rt + lo * k.ro;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (j < live && v < n && r[(li + v) * k.ri]) cuts |= uint64_t(1) << (j * V + v);
            }
        }
        // the chunk's map
        Map<V> m;
        m.none();
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t cut = uint32_t(cuts >> (j * V)) & ((1u << V) - 1);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[j][v] = rz[j][v];
                b[j][v] = rb[j][v];
                if constexpr (GATE) {
                    f[j][v] = gate_share(f[j][v]);
                    if constexpr (!BACK) {
                        b[j][v] *= gate_u(f[j][v]);
                        f[j][v] = gate_f(f[j][v]);
                    }
                }
                const float fv = BACK && GATE ? gate_f(f[j][v]) : f[j][v];
                // backwards b holds dh, and the map is f (dh + s)
                const float in = BACK ? fv * b[j][v] : b[j][v];
                const bool reset = (cut >> v) & 1;
                if (j < live) {
                    m.b[v] = reset ? (BACK ? 0.0f : in) : fv * m.b[v] + in;
                    m.a[v] *= fv;
                }
            }
            m.cut |= cut;
        }
        // joined over the wave's chunks, then over the waves
        float enter[V];
        if (chunks == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) enter[v] = state[v], state[v] = m.of(v, state[v]);
            m.after(all);
            all = m;
        } else {
            for (int d = lanes; d < kWave; d <<= 1) {
                const Map<V> up = map_up(m, d);
                if (lane >= d) m.after(up);
            }
            // a wave holds `lanes` groups, or 64 of them
            if (lane >= kWave - lanes) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    total[turn][w][0][v][lane] = m.a[v];
                    total[turn][w][1][v][lane] = m.b[v];
                }
                total_cut[turn][w][lane] = m.cut;
            }
            Map<V> before;
            before.none();
            if (lanes < kWave) {
                const Map<V> up = map_up(m, lanes);
                if (lane >= lanes) before = up;
            }
            __syncthreads();
            const int apart = lanes <= kWave ? 1 : lanes / kWave, mine = lanes < kWave ? kWave - lanes + g : lane;
            const int from = lanes <= kWave ? 0 : w & (apart - 1);
            for (int q = from; q < kWaves; q += apart) {
                Map<V> t;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    t.a[v] = total[turn][q][0][v][mine];
                    t.b[v] = total[turn][q][1][v][mine];
                }
                t.cut = total_cut[turn][q][mine];
                if (q == w) {
#pragma unroll
                    for (int v = 0; v < V; ++v) enter[v] = before.of(v, state[v]);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) state[v] = t.of(v, state[v]);
                t.after(all);
                all = t;
            }
        }
        if (first_launch) {
            if constexpr (STAGED) __syncthreads();                    // the tile is read
            continue;
        }
        // the steps again, from the state that enters the chunk
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (j < live) {
                const int tj = step(j);
                const int64_t t = ta + tj;
                const uint32_t cut = uint32_t(cuts >> (j * V)) & ((1u << V) - 1);
                float r[V], r2[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const bool reset = (cut >> v) & 1;
                    if constexpr (!BACK) {
                        enter[v] = reset ? b[j][v] : f[j][v] * enter[v] + b[j][v];
                        r[v] = enter[v];
                    } else {
                        const float gr = b[j][v] + enter[v];
                        const float past = reset ? 0.0f : t > 0 ? y[j][v] : y0[v];
                        const float fv = GATE ? gate_f(f[j][v]) : f[j][v];
                        if constexpr (GATE) {
                            const float u = gate_u(f[j][v]);
                            r[v] = (past - xs[j][v]) * gr * (fv * u);
                            r2[v] = u * gr;
                        } else {
                            r[v] = past * gr;
                            r2[v] = gr;
                        }
                        enter[v] = reset ? 0.0f : fv * gr;
                    }
                }
                if constexpr (STAGED) {
                    const int s = staged_at(int(tj * k.W) + g);
                    staged[0][s] = T(r[0]);
                    if constexpr (BACK) staged[1][s] = T(r2[0]);
                } else {
                    store_n<T, V>(static_cast<T *>(k.out.p) + o * k.out.so + i + t * k.out.st, n, r);
                    if constexpr (BACK)
                        store_n<T, V>(static_cast<T *>(k.out2.p) + o * k.out2.so + i + t * k.out2.st, n, r2);
                }
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
            if (v < n) {
                k.maps[to + at + v] = all.a[v];
                k.maps[to + k.slabs * series + at + v] = all.b[v];
                k.cuts[to + at + v] = uint8_t((all.cut >> v) & 1);
            }
    } else if (k.last.p && slab == (BACK ? 0 : k.slabs - 1)) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < n) k.last.p[o * k.last.so + (i + v) * k.last.si] = state[v];
    }
}

// How a call is cut: see the top of the file.
struct Cut {
    bool staged;
    int lanes, slabs;
    int64_t groups, slab_steps;
};

template <typename T, bool BACK> constexpr int kV = sizeof(T) == 4 ? 4 : 8;
template <typename T, bool BACK> constexpr int kSteps = !BACK && sizeof(T) == 4 ? 8 : 4;
constexpr int kStagedSteps = 8;

Cut cut_of(int V, int C, int size, bool rows, int64_t T, int64_t W, int64_t O) {
    Cut k;
    // feature-major rows that are read in pieces of less than 64 bytes, unless they are short
    k.staged = !rows && W * size < 64 && T >= 64;
    if (k.staged) {
        V = 1;
        C = kStagedSteps;
    }
    int chunks = 1;
    while (chunks < 32 && int64_t(chunks) * C < T) chunks *= 2;
    k.lanes = kThreads / chunks;
    if (k.staged) {
        k.lanes = 1;
        while (k.lanes < W) k.lanes *= 2;
    }
    k.groups = k.staged ? O : O * ((W + V - 1) / V);
    const int64_t blocks = k.staged ? O : (k.groups + k.lanes - 1) / k.lanes;
    const int64_t tile = int64_t(kThreads / k.lanes) * C;
    int64_t slabs = blocks < 512 ? (1024 + blocks - 1) / blocks : 1;
    if (slabs > kSlabs) slabs = kSlabs;
    const int64_t tiles = (T + tile - 1) / tile;
    if (slabs > tiles) slabs = tiles;
    k.slab_steps = (tiles + slabs - 1) / slabs * tile;
    k.slabs = int((T + k.slab_steps - 1) / k.slab_steps);
    return k;
}

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename T, bool GATE, bool BACK>
hipError_t launch(const RecurrenceCall &c, hipStream_t s) {
    constexpr int V = kV<T, BACK>, C = kSteps<T, BACK>;
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
    const int64_t blocks = cut.staged ? O : (cut.groups + cut.lanes - 1) / cut.lanes;
    auto go = [&](const Args &a) {
        return over_blocks(blocks * cut.slabs, kThreads, [&](int64_t first, unsigned n) {
            Args b = a;
            b.first_block = first;
            if (cut.staged)
                hipLaunchKernelGGL((recurrence_kernel<T, 1, kStagedSteps, GATE, BACK, true>), dim3(n),
                                   dim3(kThreads), 0, s, b);
            else
                hipLaunchKernelGGL((recurrence_kernel<T, V, C, GATE, BACK, false>), dim3(n), dim3(kThreads), 0, s,
                                   b);
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

}  // namespace

int64_t recurrence_workspace_bytes(int dtype, bool back, bool rows, int64_t H, int64_t T, int64_t batch) {
    const int size = dtype == DARB_F32 ? 4 : 2;
    const int V = size == 4 ? kV<float, false> : kV<half_t, false>;
    const int C = size == 4 ? (back ? kSteps<float, true> : kSteps<float, false>)
                            : (back ? kSteps<half_t, true> : kSteps<half_t, false>);
    const Cut k = cut_of(V, C, size, rows, T, rows ? H : batch, rows ? batch : H);
    if (k.slabs == 1) return 0;
    const int64_t series = H * batch;
    return padded(8 * series * k.slabs) + padded(4 * series) + padded(series * k.slabs);
}

hipError_t launch_recurrence(const RecurrenceCall &c, hipStream_t s) {
    return with_type(c.dtype, [&](auto t) {
        using T = decltype(t);
        const bool gate = c.form == DARB_RECURRENCE_GATE;
        if (c.back) return gate ? launch<T, true, true>(c, s) : launch<T, false, true>(c, s);
        return gate ? launch<T, true, false>(c, s) : launch<T, false, false>(c, s);
    });
}

}  // namespace darb
