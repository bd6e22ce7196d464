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
    const int w = threadIdx.x / kWave, lane = lane_id();
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
    const int w = threadIdx.x / kWave, lane = lane_id();
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

struct GradArgs {
    const uint32_t *starts;
    const Entry *entries;
    const void *values;
    const void *X;
    const float *dY;
    float *dvalues, *dX;
    int64_t N, B, ldx, ldy, lddx;
    int wdtype, xdtype;
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
    const int w = threadIdx.x / kWave, lane = lane_id();
    const int group = lane / LPE, in = lane % LPE;
    // Workgroups go to the 8 XCDs in turn, each with an L2 of its own, and a row's neighbouring
    // slots lie in neighbouring columns: an XCD takes columns side by side, so that a cache line
    // of values or of dvalues is its alone.
    const int64_t xcd = blockIdx.x % 8, whole = gridDim.x / 8, more = gridDim.x % 8;
    const int64_t block = xcd * whole + (xcd < more ? xcd : more) + blockIdx.x / 8;
    const int64_t c = block * (kWaves / KS) + w / KS;
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
    auto entry_at = [&](uint32_t i0, int q) {
        const uint32_t i = i0 + q * kGroups + group;
        return a.entries[i < end ? i : end - 1];
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
        auto turn = [&](uint32_t i0, const Entry (&e)[kAhead], auto is_ragged, auto is_last) {
            constexpr bool RAGGED = decltype(is_ragged)::value, LAST = decltype(is_last)::value;
            float v[kAhead];
            Loaded<float, V> dy[kAhead][U];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                v[q] = a.dX ? gather.value(e[q]) : 0.0f;
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
            Entry next[kAhead], e[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) next[q] = entry_at(from, q);
            for (uint32_t i0 = from; i0 < end; i0 += kTurn * KS) {
#pragma unroll
                for (int q = 0; q < kAhead; ++q) e[q] = next[q];
                if (i0 + kTurn * KS < end)
#pragma unroll
                    for (int q = 0; q < kAhead; ++q) next[q] = entry_at(i0 + kTurn * KS, q);
                if (i0 + kTurn <= end) turn(i0, e, is_ragged, std::false_type{});
                else turn(i0, e, is_ragged, std::true_type{});
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

// Waves to a column: enough to fill the card, but no more than have a few turns each.
template <int LPE, int V, int U> hipError_t launch_grad_t(const GradArgs &a, int64_t M, int64_t nnz, hipStream_t s) {
    const int64_t turn = kWave / LPE * (V * U >= 16 ? 2 : 4);
    int ks = 4;
    while (ks > 1 && (a.N * ks / 2 >= 8192 || nnz / a.N < 2 * ks * turn)) ks /= 2;
    // offsets of 32 bits, and a product of 24 bits each
    const bool wide = M >= 1 << 24 || a.ldy >= 1 << 22 || M * a.ldy >= int64_t(1) << 30 || nnz >= 1 << 30;
    auto launch = [&](auto share, auto is_wide) {
        constexpr int KS = decltype(share)::value;
        const int64_t blocks = (a.N + kWaves / KS - 1) / (kWaves / KS);
        if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((spmm_grad_kernel<LPE, V, U, KS, decltype(is_wide)::value>),
                           dim3(unsigned(blocks)), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    };
    if (wide) return launch(std::integral_constant<int, 1>{}, std::true_type{});
    if (ks == 1) return launch(std::integral_constant<int, 1>{}, std::false_type{});
    if (ks == 2) return launch(std::integral_constant<int, 2>{}, std::false_type{});
    return launch(std::integral_constant<int, 4>{}, std::false_type{});
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
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
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

hipError_t launch_spmm_grad(const darb_plan &p, const void *index, int wdtype, const void *values,
                            int xdtype, int64_t B, const void *X, int64_t ldx, const float *dY,
                            int64_t ldy, float *dvalues, float *dX, int64_t lddx, hipStream_t s) {
    const IndexParts x = parts_of(p, const_cast<void *>(index));
    const GradArgs a{x.starts, x.entries, values, X, dY, dvalues, dX,
                     p.N, B, ldx, ldy, lddx, wdtype, xdtype};
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
