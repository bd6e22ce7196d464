// The gradients of the DARB product Y = W_darb X, and the column index they run over.
//
//   dvalues[s] = sum_b dY[r, b] X[c, b]      for slot s, which keeps column c of row r
//   dX[c, b]   = sum over the slots s of column c of values[s] dY[r, b]
//
// Both sums run over the retained weights of a column c with the same two factors at hand:
// X[c, :] and the sum dX[c, :] stay in registers while the rows r of the column's weights go
// by, so each row of dY is gathered once for both.  The format stores weights by row, so an
// index lists them by column: for every weight its row and slot, columns in ascending order,
// a column's weights in storage order.  The index depends on the offsets alone; a program
// that retrains the retained values keeps it as long as the mask.
//
// Measured on MI355X, among other calls: 4096 x 9216 with 1.25 M weights, batch 64, 30.9 us (320 MB
// of dY's rows at 10.4 TB/s); 10 000 x 1500 with 1.0 M fp16 weights, batch 700, 179 us (2.8 GB at
// 17.6 TB/s in the main kernel, 17 us to lay out tiles, 14 to add the parts).  Bound by the L2s,
// from which random 256-byte rows come at 27.6 TB/s at most.  A single token takes 16.5 us in both.
// Their indexes take 225 and 124 us, once for a mask: a count, a scan by one workgroup, the placing.
#include <type_traits>

#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRange = 128;      // columns of one wave while the index is built: whole blocks
constexpr int kScanThreads = 1024;
// Elements of dY (3 MB) from which it is cut into tiles of the batch.  In one graph, whole and cut:
// 2000 rows x 160 24.7 and 33.6 us, 4096 x 160 61.9 and 72.6, 10 000 x 80 (3.1 MB) 43.9 and 51.1, but
// 2000 x 384 (2.9 MB) 78 and 52, 4096 x 384 (6 MB) 186 and 121.
constexpr int64_t kSplitFrom = (3 << 20) / 4;

struct Entry {
    uint32_t row, slot;
};

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

int64_t ranges_of(int64_t N) { return (N + kRange - 1) / kRange; }

// Row segments: about 4096 waves of (segment, column range), and a table of segments x N.
int64_t segments_of(int64_t M, int64_t N) {
    int64_t s = 4096 / ranges_of(N);
    if (s > (M + kWave - 1) / kWave) s = (M + kWave - 1) / kWave;
    return s < 1 ? 1 : s > 64 ? 64 : s;
}

// ---- the column index -----------------------------------------------------------------

// A wave walks its segment of the storage order, 64 rows of one group at a time (a lane each),
// and the blocks of its column range in them, and calls f(rank among the lanes that keep the
// same column, lanes that do, column - range start, row, slot) for every lane with a weight.
template <typename F>
__device__ __forceinline__ void for_weights(const uint8_t *__restrict__ offsets,
                                            const int32_t *__restrict__ perm,
                                            const BinTable &bins, int64_t N, int64_t begin,
                                            int64_t end, int64_t range, F &&f) {
    const int lane = lane_id();
    for (int g = 0; g < bins.nbins; ++g) {
        const int l = bins.log2b[g];
        int64_t i = bins.first_row[g];
        const int64_t stop = i + bins.rows[g] < end ? i + bins.rows[g] : end;
        if (i < begin) i = begin;
        const int64_t k0 = range * (kRange >> l);
        int64_t k1 = k0 + (kRange >> l);
        if (k1 > bins.nblk[g]) k1 = bins.nblk[g];
        for (; i < stop; i += kWave) {
            const bool live = i + lane < stop;
            const int64_t mine = live ? i + lane : stop - 1;
            const int64_t first = bins.first_elem[g] + (mine - bins.first_row[g]) * bins.nblk[g];
            const int32_t row = perm[mine];
            for (int64_t k = k0; k < k1; ++k) {
                // whatever the byte holds, the column stays inside the block and the matrix
                const int j = offsets[first + k] & ((1 << l) - 1);
                int64_t c = (k << l) + j;
                if (c >= N) c = N - 1;
                const int at = int(c - range * kRange);
                uint64_t same = __ballot(live);
                for (int bit = 0; bit < l; ++bit) {
                    const uint64_t set = __ballot((at >> bit) & 1);
                    same &= ((at >> bit) & 1) ? set : ~set;
                }
                const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
                f(live, rank, __popcll(same), at, row, first + k);
            }
        }
    }
}

// counts[segment][column]: the segment's weights in the column.
__global__ __launch_bounds__(kThreads) void count_columns_kernel(
    const uint8_t *__restrict__ offsets, const int32_t *__restrict__ perm, BinTable bins,
    int64_t M, int64_t N, int64_t segments, int64_t tasks, uint32_t *__restrict__ counts) {
    __shared__ uint32_t cnt[kWaves][kRange];
    const int w = wave_id(), lane = lane_id();
    const int64_t task = int64_t(blockIdx.x) * kWaves + w;
    if (task >= tasks) return;                       // no barrier below
    const int64_t range = task / segments, seg = task - range * segments;
    volatile uint32_t *c = cnt[w];
    c[lane] = 0;
    c[lane + kWave] = 0;
    for_weights(offsets, perm, bins, N, M * seg / segments, M * (seg + 1) / segments, range,
                [&](bool live, int rank, int n, int at, int32_t, int64_t) {
                    if (live && rank == 0) c[at] = c[at] + uint32_t(n);
                });
    for (int i = lane; i < kRange; i += kWave)
        if (range * kRange + i < N) counts[seg * N + range * kRange + i] = c[i];
}

// starts[c] = weights in columns before c (and starts[N] = all); counts become the position
// of each segment's first weight of the column.
__global__ __launch_bounds__(kScanThreads) void scan_columns_kernel(int64_t N, int64_t segments,
                                                                    uint32_t *__restrict__ counts,
                                                                    uint32_t *__restrict__ starts) {
    __shared__ uint32_t sums[kScanThreads / kWave];
    const int lane = lane_id(), w = threadIdx.x / kWave;
    uint32_t before = 0;
    for (int64_t base = 0; base < N; base += kScanThreads) {
        const int64_t c = base + threadIdx.x;
        uint32_t total = 0;
        if (c < N)
            for (int64_t s = 0; s < segments; ++s) total += counts[s * N + c];
        uint32_t incl = total;
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t o = __shfl_up(incl, d, kWave);
            if (lane >= d) incl += o;
        }
        if (lane == kWave - 1) sums[w] = incl;
        __syncthreads();
        uint32_t first = before, all = 0;
        for (int i = 0; i < kScanThreads / kWave; ++i) {
            if (i < w) first += sums[i];
            all += sums[i];
        }
        uint32_t at = first + incl - total;
        if (c < N) {
            starts[c] = at;
            for (int64_t s = 0; s < segments; ++s) {
                const uint32_t n = counts[s * N + c];
                counts[s * N + c] = at;
                at += n;
            }
        }
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) starts[N] = before;
}

// Every weight's (row, slot) at its place: the wave's running position of the column plus the
// weight's rank among the lanes, which hold rows in storage order.
__global__ __launch_bounds__(kThreads) void place_columns_kernel(
    const uint8_t *__restrict__ offsets, const int32_t *__restrict__ perm, BinTable bins,
    int64_t M, int64_t N, int64_t segments, int64_t tasks, const uint32_t *__restrict__ counts,
    Entry *__restrict__ entries) {
    __shared__ uint32_t pos[kWaves][kRange];
    const int w = wave_id(), lane = lane_id();
    const int64_t task = int64_t(blockIdx.x) * kWaves + w;
    if (task >= tasks) return;                       // no barrier below
    const int64_t range = task / segments, seg = task - range * segments;
    volatile uint32_t *p = pos[w];
    for (int i = lane; i < kRange; i += kWave)
        p[i] = range * kRange + i < N ? counts[seg * N + range * kRange + i] : 0;
    for_weights(offsets, perm, bins, N, M * seg / segments, M * (seg + 1) / segments, range,
                [&](bool live, int rank, int n, int at, int32_t row, int64_t slot) {
                    const uint32_t first = p[at];    // read by all before the first lane adds
                    if (live) entries[first + rank] = {uint32_t(row), uint32_t(slot)};
                    if (live && rank == 0) p[at] = first + uint32_t(n);
                });
}

// ---- the gradients --------------------------------------------------------------------

// Workgroups go to the 8 XCDs in turn, each with an L2 of its own: the task of workgroup i of n
// such that an XCD's tasks lie side by side.  A row's neighbouring slots lie in neighbouring
// columns, so that a cache line of values or of dvalues belongs to one XCD.
__device__ __forceinline__ int64_t side_by_side(uint32_t i, uint32_t n) {
    const uint32_t xcd = i % 8, whole = n / 8, more = n % 8;
    return int64_t(xcd) * whole + (xcd < more ? xcd : more) + i / 8;
}

struct GradArgs {
    const uint32_t *starts;
    const Entry *entries;
    const void *values;
    const void *X;
    const float *dY;
    float *dvalues, *dX;
    int64_t N, B, ldx, ldy, lddx;
    int wdtype, xdtype;
    int64_t first;                      // the launch's first column
};

// The weight's row of dY from one of the lane's columns on, and its value.  32 bits of offset
// (WIDE: 64) from bases that all lanes share.
template <bool WIDE> struct Gather {
    const GradArgs &a;
    uint32_t ld;                        // bytes of a row of dY, below 2^24 as rows are
    __device__ __forceinline__ const float *row(const Entry &e, int64_t col) const {
        if (WIDE) return a.dY + int64_t(e.row) * a.ldy + col;
        const uint32_t at = __umul24(e.row, ld) + uint32_t(col) * 4u;
        return reinterpret_cast<const float *>(reinterpret_cast<const char *>(a.dY) + at);
    }
    __device__ __forceinline__ float value(const Entry &e) const {
        const uint32_t s = e.slot;
        if (a.wdtype == DARB_F32) return WIDE ? static_cast<const float *>(a.values)[s] : at32<float>(a.values, s);
        return float(WIDE ? static_cast<const half_t *>(a.values)[s] : at32<half_t>(a.values, s));
    }
    template <typename T> __device__ __forceinline__ static T at32(const void *p, uint32_t i) {
        return *reinterpret_cast<const T *>(static_cast<const char *>(p) + i * uint32_t(sizeof(T)));
    }
};

// A workgroup takes kWaves / KS columns; KS waves share a column's weights.  LPE lanes take one
// weight, V batch columns each, U times: a wave handles 64 / LPE weights at once and
// LPE * V * U batch columns; a wider batch goes over the column's weights again for each such
// tile, adding to dvalues.  In the last tile a lane whose columns would pass the batch's end
// takes the last V instead and leaves those that the lane before has out of its dot product.
template <int LPE, int V, int U, int KS, bool WIDE>
__global__ __launch_bounds__(kThreads) void spmm_grad_kernel(GradArgs a) {
    constexpr int kGroups = kWave / LPE;      // weights at once
    constexpr int kAhead = V * U >= 16 ? 2 : 4;     // steps whose gathers are in flight together
    constexpr int kCols = LPE * V;            // batch columns of one of the U parts
    constexpr uint32_t kTurn = kGroups * kAhead;
    __shared__ float part[KS > 1 ? (KS - 1) * (kWaves / KS) : 1][KS > 1 ? kCols * U : 1];
    const int w = wave_id(), lane = lane_id();
    const int group = lane / LPE, in = lane % LPE;
    const int64_t block = side_by_side(blockIdx.x, gridDim.x);
    const int64_t c = a.first + block * (kWaves / KS) + w / KS;
    const int share = w % KS;
    const bool has = c < a.N;
    uint32_t begin = 0, end = 0;
    if (has) {
        begin = __builtin_amdgcn_readfirstlane(a.starts[c]);
        end = __builtin_amdgcn_readfirstlane(a.starts[c + 1]);
    }
    const Gather<WIDE> gather{a, uint32_t(a.ldy) * 4u};
    // The waves take turns of kAhead steps, so that the waves of all columns, which hold rows in
    // one order, go through the same part of dY at about the same time.
    const uint32_t from = begin + share * kTurn;
    // A turn's weights, past the end the last one again.  Where it has no more than a wave has
    // lanes, each lane reads one and its value, and the groups fetch theirs through LDS: read from
    // memory by all lanes of a group they would cost the L1 as much as the rows of dY.
    constexpr bool kSpread = LPE > 1 && kTurn <= kWave;
    struct Weights {
        Entry e[kSpread ? 1 : kAhead];
        float v[kSpread ? 1 : kAhead];
    };
    auto load_weights = [&](uint32_t i0, Weights &t) {
#pragma unroll
        for (int q = 0; q < (kSpread ? 1 : kAhead); ++q) {
            const uint32_t i = kSpread ? i0 + lane % kTurn : i0 + q * kGroups + group;
            t.e[q] = a.entries[i < end ? i : end - 1];
        }
    };
    auto load_values = [&](Weights &t) {
#pragma unroll
        for (int q = 0; q < (kSpread ? 1 : kAhead); ++q) t.v[q] = a.dX ? gather.value(t.e[q]) : 0.0f;
    };
    auto spread = [&](const Weights &t, Entry (&e)[kAhead], float (&v)[kAhead]) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            if constexpr (kSpread) {
                const int from_lane = q * kGroups + group;
                e[q] = {__shfl(t.e[0].row, from_lane, kWave), __shfl(t.e[0].slot, from_lane, kWave)};
                v[q] = __shfl(t.v[0], from_lane, kWave);
            } else {
                e[q] = t.e[q];
                v[q] = t.v[q];
            }
        }
    };
    for (int64_t tile = 0; tile < a.B; tile += int64_t(kCols) * U) {
        float x[U][V], acc[U][V];
        int64_t col[U];
        int skip[U];
        const bool ragged = tile + kCols * U > a.B;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t own = tile + u * kCols + in * V;
            col[u] = own + V <= a.B ? own : a.B - V;
            skip[u] = own - col[u] < V ? int(own - col[u]) : V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                acc[u][i] = 0.0f;
                x[u][i] = 0.0f;
                if (has && a.dvalues) {
                    const int64_t at = c * a.ldx + col[u] + i;
                    x[u][i] = a.xdtype == DARB_F32 ? static_cast<const float *>(a.X)[at]
                                                   : float(static_cast<const half_t *>(a.X)[at]);
                }
            }
        }
        // one turn; RAGGED: the batch may end in it, LAST: the weights may
        auto turn = [&](uint32_t i0, const Entry (&e)[kAhead], const float (&v)[kAhead], auto is_ragged, auto is_last) {
            constexpr bool RAGGED = decltype(is_ragged)::value, LAST = decltype(is_last)::value;
            Loaded<float, V> dy[kAhead][U];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const float *row = gather.row(e[q], col[0]);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    dy[q][u] = load_vec<float, V>(RAGGED ? gather.row(e[q], col[u]) : row + u * kCols);
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const bool live = !LAST || i0 + q * kGroups + group < end;
                float dot = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float to = fmaf(v[q], dy[q][u][i], acc[u][i]);
                        acc[u][i] = live ? to : acc[u][i];
                        if (!RAGGED || i >= skip[u]) dot = fmaf(x[u][i], dy[q][u][i], dot);
                    }
                dot = group_reduce<LPE, AddOp>(dot);
                if (a.dvalues && live && in == 0) {
                    float *to = WIDE ? a.dvalues + e[q].slot
                                     : reinterpret_cast<float *>(reinterpret_cast<char *>(a.dvalues) + e[q].slot * 4u);
                    *to = tile == 0 ? dot : *to + dot;
                }
            }
        };
        auto weights = [&](auto is_ragged) {
            if (from >= end) return;
            Entry e[kAhead];
            float v[kAhead];
            Weights next;
            load_weights(from, next);
            load_values(next);
            for (uint32_t i0 = from; i0 < end; i0 += kTurn * KS) {
                spread(next, e, v);
                if (i0 + kTurn * KS < end) load_weights(i0 + kTurn * KS, next);
                if (i0 + kTurn <= end) turn(i0, e, v, is_ragged, std::false_type{});
                else turn(i0, e, v, is_ragged, std::true_type{});
                if (i0 + kTurn * KS < end) load_values(next);
            }
        };
        if (ragged) weights(std::true_type{});
        else weights(std::false_type{});
        if (!a.dX) continue;
        // the groups' sums, then the waves', in a fixed order
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = acc[u][i];
                for (int d = LPE; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
                acc[u][i] = s;
            }
        if constexpr (KS > 1) {
            if (share > 0 && group == 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        part[(w / KS) * (KS - 1) + share - 1][u * kCols + in * V + i] = acc[u][i];
            }
            __syncthreads();
            if (share == 0 && group == 0)
                for (int k = 0; k < KS - 1; ++k)
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            acc[u][i] += part[(w / KS) * (KS - 1) + k][u * kCols + in * V + i];
            __syncthreads();
        }
        if (has && share == 0 && group == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (tile + u * kCols + in * V < a.B) store_vec<float, V>(a.dX + c * a.lddx + col[u], acc[u]);
        }
    }
}

// Waves to a column: enough to fill the card, 8192 in all, but no more than have a few turns each.
// (4096, 8192 and 16 384, in one graph: 9216 columns of 128 weights at batch 64 29.9, 29.4 and 34.2
// us, 6000 of 256 at batch 128 62.9, 57.5 and 65.2, though at batch 256 104, 115 and 128; 20 000 of 128
// at batch 64 56.5 all three, 67.3 with 32 768.)
int waves_of(int64_t N, int64_t nnz, int64_t turn) {
    int ks = 4;
    while (ks > 1 && (N * ks / 2 >= 8192 || nnz / N < 2 * ks * turn)) ks /= 2;
    return ks;
}

// f(first column, workgroups) for every launch over the columns: below 2^32 threads, also where it
// has kSplitTiles times as many workgroups.
template <int KS, typename F> hipError_t over_columns(int64_t N, F &&f) {
    constexpr int64_t kEach = kWaves / KS, kMost = (int64_t(1) << 19) * kEach;
    for (int64_t first = 0; first < N; first += kMost) {
        const int64_t n = N - first < kMost ? N - first : kMost;
        const hipError_t e = f(first, uint32_t((n + kEach - 1) / kEach));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int LPE, int V, int U> hipError_t launch_grad_t(const GradArgs &a, int64_t M, int64_t nnz, hipStream_t s) {
    const int ks = waves_of(a.N, nnz, kWave / LPE * (V * U >= 16 ? 2 : 4));
    // offsets of 32 bits, and a product of 24 bits each
    const bool wide = M >= 1 << 24 || a.ldy >= 1 << 22 || M * a.ldy >= int64_t(1) << 30 || nnz >= 1 << 30;
    auto launch = [&](auto share, auto is_wide) {
        constexpr int KS = decltype(share)::value;
        return over_columns<KS>(a.N, [&](int64_t first, uint32_t blocks) {
            GradArgs part = a;
            part.first = first;
            hipLaunchKernelGGL((spmm_grad_kernel<LPE, V, U, KS, decltype(is_wide)::value>),
                               dim3(blocks), dim3(kThreads), 0, s, part);
            return hipGetLastError();
        });
    };
    if (wide) return launch(std::integral_constant<int, 1>{}, std::true_type{});
    if (ks == 1) return launch(std::integral_constant<int, 1>{}, std::false_type{});
    if (ks == 2) return launch(std::integral_constant<int, 2>{}, std::false_type{});
    return launch(std::integral_constant<int, 4>{}, std::false_type{});
}

// ---- a dY too large for the L2s --------------------------------------------------------
//
// Gathers of dY's rows run at the L2's rate only while what they gather from stays in an XCD's
// 4 MB.  A larger dY is copied into tiles of 64 batch columns, [tile][M][64] (a row 256 aligned
// bytes, zeros past the batch), the weights' values into the index' order beside their rows, and
// each XCD goes through tile after tile.  A tile's part of dvalues lies in the index' order too;
// the parts are added, slot by slot, at the end.

constexpr int kSplitCols = 64;
constexpr int kSplitTiles = 16;         // tiles of a launch, at most: what bounds the workspace

struct Pair {
    uint32_t row;
    float value;
};

struct SplitArgs {
    GradArgs g;
    Pair *pairs;
    float *tiles;                       // [tiles][M][kSplitCols]
    float *parts;                       // [tiles][nnz]
    int64_t M, nnz, first_tile;
    uint32_t blocks;                    // workgroups of a tile
};

__device__ __forceinline__ void pair_values(const SplitArgs &a, uint32_t block, uint32_t blocks) {
    const int64_t i = side_by_side(block, blocks) * kThreads + threadIdx.x;
    if (i >= a.nnz) return;
    const Entry e = a.g.entries[i];
    float v = 0.0f;
    if (a.g.dX) v = a.g.wdtype == DARB_F32 ? static_cast<const float *>(a.g.values)[e.slot]
                                           : float(static_cast<const half_t *>(a.g.values)[e.slot]);
    a.pairs[i] = {e.row, v};
}

// The first pair_blocks workgroups gather the weights' values while the others copy the tiles, a
// thread four columns of a row: one waits for latency, the other for bandwidth.
__global__ __launch_bounds__(kThreads) void tile_rows_kernel(SplitArgs a, uint32_t pair_blocks, uint32_t row_blocks) {
    constexpr int kPerRow = kSplitCols / 4;
    if (blockIdx.x < pair_blocks) {
        pair_values(a, blockIdx.x, pair_blocks);
        return;
    }
    const uint32_t block = blockIdx.x - pair_blocks, tile = block / row_blocks;
    const int64_t i = int64_t(block - tile * row_blocks) * kThreads + threadIdx.x, r = i / kPerRow;
    if (r >= a.M) return;
    const int64_t c = (a.first_tile + tile) * kSplitCols + i % kPerRow * 4;
    const float *from = a.g.dY + r * a.g.ldy + c;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c + 4 <= a.g.B) {
        const Loaded<float, 4> v = load_vec<float, 4>(from);
        x = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        if (c < a.g.B) x.x = from[0];
        if (c + 1 < a.g.B) x.y = from[1];
        if (c + 2 < a.g.B) x.z = from[2];
    }
    reinterpret_cast<float4 *>(a.tiles)[(tile * a.M + r) * kPerRow + i % kPerRow] = x;
}

// As spmm_grad_kernel with 8 lanes to a weight, 8 batch columns each.
template <int KS>
__global__ __launch_bounds__(kThreads) void split_grad_kernel(SplitArgs a) {
    constexpr int LPE = 8, U = 2, V = 4, kGroups = kWave / LPE, kAhead = 4;
    constexpr uint32_t kTurn = kGroups * kAhead;
    __shared__ float part[KS > 1 ? (KS - 1) * (kWaves / KS) : 1][kSplitCols];
    const int w = wave_id(), lane = lane_id(), group = lane / LPE, in = lane % LPE;
    const int64_t task = side_by_side(blockIdx.x, gridDim.x);
    const int64_t t = task / a.blocks, c = a.g.first + (task - t * a.blocks) * (kWaves / KS) + w / KS;
    const int share = w % KS;
    const bool has = c < a.g.N;
    uint32_t begin = 0, end = 0;
    if (has) {
        begin = __builtin_amdgcn_readfirstlane(a.g.starts[c]);
        end = __builtin_amdgcn_readfirstlane(a.g.starts[c + 1]);
    }
    const int64_t col0 = (a.first_tile + t) * kSplitCols + in * V;
    float x[U][V], acc[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t col = col0 + u * (LPE * V) + i;
            acc[u][i] = x[u][i] = 0.0f;
            if (has && a.parts && col < a.g.B)
                x[u][i] = a.g.xdtype == DARB_F32 ? static_cast<const float *>(a.g.X)[c * a.g.ldx + col]
                                                 : float(static_cast<const half_t *>(a.g.X)[c * a.g.ldx + col]);
        }
    const char *tile = reinterpret_cast<const char *>(a.tiles + t * a.M * kSplitCols);
    float *parts = a.parts ? a.parts + t * a.nnz : nullptr;
    const uint32_t from = begin + share * kTurn;
    // A turn's weights, a lane each (past the end the last one again), which their groups then
    // fetch through LDS: read from memory by all lanes of a group they would cost the L1 as much
    // as the rows of dY.
    static_assert(kTurn <= kWave, "a lane per weight");
    auto load_pair = [&](uint32_t i0) {
        const uint32_t i = i0 + lane % kTurn;
        return a.pairs[i < end ? i : end - 1];
    };
    auto spread = [&](const Pair &mine, Pair (&e)[kAhead]) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            e[q].row = __shfl(mine.row, q * kGroups + group, kWave);
            e[q].value = __shfl(mine.value, q * kGroups + group, kWave);
        }
    };
    auto turn = [&](uint32_t i0, const Pair (&e)[kAhead], auto is_last) {
        constexpr bool LAST = decltype(is_last)::value;
        Loaded<float, V> dy[kAhead][U];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const uint32_t at = (e[q].row << 8) + uint32_t(in) * 16u;       // rows below 2^24
#pragma unroll
            for (int u = 0; u < U; ++u)
                dy[q][u] = load_vec<float, V>(reinterpret_cast<const float *>(tile + at) + u * (LPE * V));
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const bool live = !LAST || i0 + q * kGroups + group < end;
            float dot = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float to = fmaf(e[q].value, dy[q][u][j], acc[u][j]);
                    acc[u][j] = live ? to : acc[u][j];
                    dot = fmaf(x[u][j], dy[q][u][j], dot);
                }
            dot = group_reduce<LPE, AddOp>(dot);
            if (parts && live && in == 0) (parts + i0)[q * kGroups + group] = dot;
        }
    };
    if (from < end) {
        Pair next = load_pair(from), e[kAhead];
        for (uint32_t i0 = from; i0 < end; i0 += kTurn * KS) {
            spread(next, e);
            if (i0 + kTurn * KS < end) next = load_pair(i0 + kTurn * KS);
            if (i0 + kTurn <= end) turn(i0, e, std::false_type{});
            else turn(i0, e, std::true_type{});
        }
    }
    if (!a.g.dX) return;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float s = acc[u][j];
            for (int d = LPE; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
            acc[u][j] = s;
        }
    if constexpr (KS > 1) {
        if (share > 0 && group == 0)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    part[(w / KS) * (KS - 1) + share - 1][u * (LPE * V) + in * V + j] = acc[u][j];
        __syncthreads();
        if (share == 0 && group == 0)
            for (int k = 0; k < KS - 1; ++k)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        acc[u][j] += part[(w / KS) * (KS - 1) + k][u * (LPE * V) + in * V + j];
    }
    if (has && share == 0 && group == 0)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t col = col0 + u * (LPE * V);
            float *to = a.g.dX + c * a.g.lddx + col;
            if (col + V <= a.g.B) {
                store_vec<float, V>(to, acc[u]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (col + j < a.g.B) to[j] = acc[u][j];
            }
        }
}

// dvalues from the tiles' parts, added to what earlier tiles left where there were any.
__global__ __launch_bounds__(kThreads) void sum_parts_kernel(const float *__restrict__ parts, int64_t nnz, int tiles,
                                                             const Entry *__restrict__ entries, bool add,
                                                             float *__restrict__ dvalues) {
    const int64_t i = side_by_side(blockIdx.x, gridDim.x) * kThreads + threadIdx.x;
    if (i >= nnz) return;
    const uint32_t slot = entries[i].slot;
    float s = add ? dvalues[slot] : 0.0f;
    int t = 0;
    for (; t + 8 <= tiles; t += 8) {                 // loads side by side
        float x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = parts[(t + q) * nnz + i];
#pragma unroll
        for (int q = 0; q < 8; ++q) s += x[q];
    }
#pragma unroll 4
    for (; t < tiles; ++t) s += parts[t * nnz + i];
    dvalues[slot] = s;
}

bool is_split(int64_t M, int64_t B) { return B > kSplitCols && M < 1 << 24 && M * B > kSplitFrom; }

struct SplitRoom {
    int64_t tiles, pairs_at, tiles_at, parts_at, bytes;
};

SplitRoom split_room(const darb_plan &p, int64_t B) {
    SplitRoom r;
    r.tiles = (B + kSplitCols - 1) / kSplitCols;
    const int64_t at_once = r.tiles < kSplitTiles ? r.tiles : kSplitTiles;
    r.pairs_at = 0;
    r.tiles_at = padded(p.nnz * int64_t(sizeof(Pair)));
    r.parts_at = r.tiles_at + padded(at_once * p.M * kSplitCols * 4);
    r.bytes = r.parts_at + padded(at_once * p.nnz * 4);
    return r;
}

hipError_t launch_split(const darb_plan &p, const GradArgs &g, void *workspace, hipStream_t s) {
    const SplitRoom r = split_room(p, g.B);
    char *w = static_cast<char *>(workspace);
    SplitArgs a{g, reinterpret_cast<Pair *>(w + r.pairs_at), reinterpret_cast<float *>(w + r.tiles_at),
                g.dvalues ? reinterpret_cast<float *>(w + r.parts_at) : nullptr, p.M, p.nnz, 0, 0};
    const dim3 each(unsigned((p.nnz + kThreads - 1) / kThreads));
    const int ks = waves_of(p.N, p.nnz, 32);
    // a launch has below 2^32 threads
    const uint32_t row_blocks = uint32_t((p.M * (kSplitCols / 4) + kThreads - 1) / kThreads);
    int64_t most = ((int64_t(1) << 24) - 1 - each.x) / row_blocks;
    if (most > kSplitTiles) most = kSplitTiles;
    auto columns = [&](auto share, int64_t n) {
        constexpr int KS = decltype(share)::value;
        return over_columns<KS>(p.N, [&](int64_t first, uint32_t blocks) {
            a.g.first = first;
            a.blocks = blocks;
            hipLaunchKernelGGL((split_grad_kernel<KS>), dim3(unsigned(blocks * n)), dim3(kThreads), 0, s, a);
            return hipGetLastError();
        });
    };
    for (a.first_tile = 0; a.first_tile < r.tiles; a.first_tile += most) {
        const int64_t n = r.tiles - a.first_tile < most ? r.tiles - a.first_tile : most;
        const uint32_t pair_blocks = a.first_tile == 0 ? each.x : 0;
        hipLaunchKernelGGL(tile_rows_kernel, dim3(pair_blocks + row_blocks * uint32_t(n)), dim3(kThreads), 0, s, a,
                           pair_blocks, row_blocks);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (ks == 1) e = columns(std::integral_constant<int, 1>{}, n);
        else if (ks == 2) e = columns(std::integral_constant<int, 2>{}, n);
        else e = columns(std::integral_constant<int, 4>{}, n);
        if (e != hipSuccess) return e;
        if (g.dvalues)
            hipLaunchKernelGGL(sum_parts_kernel, each, dim3(kThreads), 0, s, a.parts, p.nnz, int(n),
                               g.entries, a.first_tile > 0, g.dvalues);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

struct IndexParts {
    uint32_t *starts;
    Entry *entries;
    uint32_t *counts;
};

IndexParts parts_of(const darb_plan &p, void *index) {
    char *b = static_cast<char *>(index);
    const int64_t at = padded((p.N + 1) * 4), counts = at + padded(p.nnz * int64_t(sizeof(Entry)));
    return {reinterpret_cast<uint32_t *>(b), reinterpret_cast<Entry *>(b + at),
            reinterpret_cast<uint32_t *>(b + counts)};
}

}  // namespace

int64_t transpose_bytes(const darb_plan &p) {
    return padded((p.N + 1) * 4) + padded(p.nnz * int64_t(sizeof(Entry))) +
           padded(segments_of(p.M, p.N) * p.N * 4);
}

hipError_t launch_transpose(const darb_plan &p, const uint8_t *offsets, void *index, hipStream_t s) {
    const IndexParts x = parts_of(p, index);
    const int64_t segments = segments_of(p.M, p.N), tasks = segments * ranges_of(p.N);
    const int64_t blocks = (tasks + kWaves - 1) / kWaves;
    if (blocks >= 1 << 24) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(count_columns_kernel, dim3(unsigned(blocks)), dim3(kThreads), 0, s, offsets,
                       p.d_perm, p.bins, p.M, p.N, segments, tasks, x.counts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(scan_columns_kernel, dim3(1), dim3(kScanThreads), 0, s, p.N, segments,
                       x.counts, x.starts);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(place_columns_kernel, dim3(unsigned(blocks)), dim3(kThreads), 0, s, offsets,
                       p.d_perm, p.bins, p.M, p.N, segments, tasks, x.counts, x.entries);
    return hipGetLastError();
}

int64_t spmm_grad_workspace_bytes(const darb_plan &p, int64_t B) {
    return is_split(p.M, B) ? split_room(p, B).bytes : 0;
}

hipError_t launch_spmm_grad(const darb_plan &p, const void *index, int wdtype, const void *values,
                            int xdtype, int64_t B, const void *X, int64_t ldx, const float *dY,
                            int64_t ldy, float *dvalues, float *dX, int64_t lddx, void *workspace,
                            hipStream_t s) {
    const IndexParts x = parts_of(p, const_cast<void *>(index));
    const GradArgs a{x.starts, x.entries, values, X, dY, dvalues, dX, p.N, B, ldx, ldy, lddx, wdtype, xdtype, 0};
    if (is_split(p.M, B)) return launch_split(p, a, workspace, s);
    // 16 bytes a lane and few lanes to a weight, so that a wave has many weights' rows under way.
    // (4096 x 9216 with 1.2 M weights, so and with twice the lanes or a column a lane: batch 16 18.6 and
    // 27.0 us, 32 21.2 and 22.2, 64 29.4 and 38.0, 192 65.1 and 84.6, though 128 52.5 and 48.8; 2000 x
    // 3000: batch 8 8.8 and 10.0, 32 10.1 and 11.6, 128 19.9 and 20.8.)
    if (B == 1) return launch_grad_t<1, 1, 1>(a, p.M, p.nnz, s);
    if (B < 4) return launch_grad_t<4, 1, 1>(a, p.M, p.nnz, s);
    if (B == 4) return launch_grad_t<1, 4, 1>(a, p.M, p.nnz, s);
    if (B <= 8) return launch_grad_t<2, 4, 1>(a, p.M, p.nnz, s);
    if (B <= 16) return launch_grad_t<4, 4, 1>(a, p.M, p.nnz, s);
    if (B <= 32) return launch_grad_t<4, 4, 2>(a, p.M, p.nnz, s);
    if (B <= 64) return launch_grad_t<8, 4, 2>(a, p.M, p.nnz, s);
    if (B <= 128) return launch_grad_t<8, 4, 4>(a, p.M, p.nnz, s);
    if (B <= 192) return launch_grad_t<16, 4, 3>(a, p.M, p.nnz, s);
    return launch_grad_t<16, 4, 4>(a, p.M, p.nnz, s);
}

}  // namespace darb
