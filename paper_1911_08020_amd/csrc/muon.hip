// The orthogonalised update of weight matrices.
//
//   u = the gradient, or mu m + (1 - mu) g after m = mu m + (1 - mu) g  (or m itself)
//   X = u / (|u| + eps)  (Frobenius norm),  then `steps` times, with A = X X^T,
//   X = a X + (b A + c A A) X;   (a, b, c) = (3.4445, -4.7750, 2.0315)
//   p = p keep - scale X, or X itself
//
// The quintic p(s) = a s + b s^3 + c s^5 maps [0, 1.21] into itself and its steps take the singular
// values from 0.01 up to between 0.68 and 1.21; the singular vectors stay.  X is held with its
// shorter side m as rows.  A and b A + c A A are symmetric: only tiles on and below the diagonal
// are computed, and written to both places.
//
// The products run on the matrix cores in fp16 with fp32 sums.  A matrix is kept as hi + lo, two
// fp16 parts of its value times a power of two (22 bits; the greatest values, |x| <= 1.21,
// |A| <= 1.46 and |b A + c A A| <= 2.81, stay in fp16's range), and a product as accurate as fp32
// is hi hi + hi lo + lo hi.  A result of 16 bits takes hi hi alone for A and for the last product:
// each element is then off by at most 2^-11 of itself, the result by 1 to 3 10^-3 of its norm (the
// steps amplify what happens to small singular values as they do these), beside a rounding of
// 2^-9.  A A is computed from both parts then too: A is close to a multiple of the identity
// when m is well below n, and its one large diagonal's rounding would be half of the error.  a X is
// added from both parts, so that what X has in no direction does not grow out of its rounding.
//
// Every product is rows by rows, C[i, j] = sum_k P[i, k] Q[j, k]: A from X, A A from A
// (symmetric), and the last one from b A + c A A and X^T, so each step writes X in both
// orders.  Buffers are padded with zeros to whole tiles, which the steps keep, so that no product
// checks a bound.  All matrices of a call go through one launch per product.
#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 0x1p15f, kScaleB = 0x1p14f;       // of X and A; of b A + c A A
constexpr int kNormBlocks = 256;        // at most, a matrix
constexpr int kNormTile = 8192;
constexpr int kNormThreads = 256;
constexpr int kCutTile = 64;
constexpr int kDepth = 32;              // columns of P and Q in LDS at a time

typedef half_t Half4 __attribute__((ext_vector_type(4)));
typedef half_t Half8 __attribute__((ext_vector_type(8)));
typedef float Float4 __attribute__((ext_vector_type(4)));

// A matrix's buffers, in halves from its base.
struct Places {
    int64_t mn, mm;
    __host__ __device__ Places(const MuonTensor &t) : mn(int64_t(t.m) * t.n), mm(int64_t(t.m) * t.m) {}
    // X [m x n] and X^T [n x m] of step `at`, hi and lo
    __host__ __device__ int64_t x(int at, int lo) const { return (4 * (at & 1) + lo) * mn; }
    __host__ __device__ int64_t xt(int at, int lo) const { return (4 * (at & 1) + 2 + lo) * mn; }
    __host__ __device__ int64_t a(int lo) const { return 8 * mn + lo * mm; }
    __host__ __device__ int64_t b(int lo) const { return 8 * mn + (2 + lo) * mm; }
    __host__ __device__ int64_t all() const { return 8 * mn + 4 * mm; }
};

// The partial sums of every matrix lie before the matrices.
__host__ __device__ constexpr int64_t norms_bytes() { return int64_t(kMuonTensors) * kNormBlocks * 8; }

__device__ __forceinline__ half_t *matrices(const MuonCall &c, const MuonTensor &t) {
    return reinterpret_cast<half_t *>(static_cast<char *>(c.workspace) + norms_bytes()) + t.base;
}

__device__ __forceinline__ float load_typed(int type, const void *p, int64_t at) {
    if (type == DARB_F32) return static_cast<const float *>(p)[at];
    if (type == DARB_F16) return float(static_cast<const half_t *>(p)[at]);
    return float(static_cast<const bf16_t *>(p)[at]);
}

__device__ __forceinline__ void store_typed(int type, void *p, int64_t at, float x) {
    if (type == DARB_F32) static_cast<float *>(p)[at] = x;
    else if (type == DARB_F16) static_cast<half_t *>(p)[at] = half_t(x);
    else static_cast<bf16_t *>(p)[at] = bf16_t(x);
}

// ---- momentum and norm -----------------------------------------------------------------

__host__ __device__ __forceinline__ int norm_blocks(const MuonTensor &t) {
    const int64_t tiles = (int64_t(t.rows) * t.cols + kNormTile - 1) / kNormTile;
    return int(tiles < kNormBlocks ? tiles : kNormBlocks);
}

__global__ __launch_bounds__(kNormThreads) void norm_kernel(MuonCall c) {
    __shared__ double room[kNormThreads / kWave];
    const int which = int(blockIdx.y);
    const MuonTensor &t = c.t[which];
    const int blocks = norm_blocks(t);
    if (int(blockIdx.x) >= blocks) return;
    const float gs = c.grad_scale ? *c.grad_scale : 1.0f;
    const int64_t n = int64_t(t.rows) * t.cols;
    double sum = 0.0;
    for (int64_t e = int64_t(blockIdx.x) * kNormThreads + threadIdx.x; e < n; e += int64_t(blocks) * kNormThreads) {
        const int64_t at = t.ld_in == t.cols ? e : e / t.cols * t.ld_in + e % t.cols;
        float u = load_typed(t.gdtype, t.grad, at) * gs;
        if (t.momentum) {
            const float m = c.mu * t.momentum[e] + c.one_mu * u;
            t.momentum[e] = m;
            u = c.nesterov ? c.mu * m + c.one_mu * u : m;
        }
        sum += double(u) * double(u);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane_id() == 0) room[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / kWave; ++w) sum += room[w];
        static_cast<double *>(c.workspace)[which * kNormBlocks + blockIdx.x] = sum;
    }
}

// ---- X of the first step ---------------------------------------------------------------

struct Split {
    half_t hi, lo;
};
__device__ __forceinline__ Split split(float scaled) {
    const half_t hi = half_t(scaled);
    return {hi, half_t(scaled - float(hi))};
}

// Padded to whole tiles of the natural orientation.
__host__ __device__ __forceinline__ int padded_rows(const MuonTensor &t) { return t.rows <= t.cols ? t.m : t.n; }
__host__ __device__ __forceinline__ int padded_cols(const MuonTensor &t) { return t.rows <= t.cols ? t.n : t.m; }

__global__ __launch_bounds__(256) void cut_kernel(MuonCall c, int first_block) {
    __shared__ float tile[kCutTile][kCutTile + 1];
    __shared__ double room[256 / kWave];
    int block = first_block + int(blockIdx.x), which = 0;
    for (;; ++which) {
        const int blocks = (padded_rows(c.t[which]) / kCutTile) * (padded_cols(c.t[which]) / kCutTile);
        if (block < blocks) break;
        block -= blocks;
    }
    const MuonTensor &t = c.t[which];
    const int tid = int(threadIdx.x), R = padded_rows(t), C = padded_cols(t);
    const int r0 = block / (C / kCutTile) * kCutTile, c0 = block % (C / kCutTile) * kCutTile;
    double sum = tid < norm_blocks(t) ? static_cast<const double *>(c.workspace)[which * kNormBlocks + tid] : 0.0;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane_id() == 0) room[wave_id()] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < 256 / kWave; ++w) sum += room[w];
    const double inverse = double(kScaleX) / (sqrt(sum) + c.eps);
    const float gs = c.grad_scale ? *c.grad_scale : 1.0f;
    half_t *base = matrices(c, t);
    const Places at(t);
    const bool turned = t.rows > t.cols;                    // X is u^T
    half_t *nh = base + (turned ? at.xt(0, 0) : at.x(0, 0)), *nl = base + (turned ? at.xt(0, 1) : at.x(0, 1));
    half_t *fh = base + (turned ? at.x(0, 0) : at.xt(0, 0)), *fl = base + (turned ? at.x(0, 1) : at.xt(0, 1));
    const int col = tid % kCutTile;
    for (int row = tid / kCutTile; row < kCutTile; row += 256 / kCutTile) {
        const int r = r0 + row, q = c0 + col;
        float x = 0.0f;
        if (r < t.rows && q < t.cols) {
            float u = load_typed(t.gdtype, t.grad, r * t.ld_in + q) * gs;
            if (t.momentum) {
                const float m = t.momentum[int64_t(r) * t.cols + q];
                u = c.nesterov ? c.mu * m + c.one_mu * u : m;
            }
            x = float(double(u) * inverse);
        }
        tile[row][col] = x;
        const Split s = split(x);
        nh[int64_t(r) * C + q] = s.hi;
        nl[int64_t(r) * C + q] = s.lo;
    }
    __syncthreads();
    for (int row = tid / kCutTile; row < kCutTile; row += 256 / kCutTile) {
        const Split s = split(tile[col][row]);
        fh[int64_t(c0 + row) * R + r0 + col] = s.hi;
        fl[int64_t(c0 + row) * R + r0 + col] = s.lo;
    }
}

// ---- the products ----------------------------------------------------------------------

enum { kGram, kSquare, kApply, kResult };                   // A; b A + c A A; X; the last X

// Tiles on and below the diagonal of q x q, or all of them.
__host__ __device__ __forceinline__ int tiles_of(const MuonTensor &t, int mode, int tile) {
    const int q = t.m / tile;
    return mode == kGram || mode == kSquare ? q * (q + 1) / 2 : q * (t.n / tile);
}

// Place of a 16-byte piece in its row of kDepth halves: rows that a read takes together use
// different banks.
__device__ __forceinline__ int piece(int row, int k) { return k ^ ((row >> 1 & 3) ^ (row >> 3 & 1)); }

typedef __attribute__((address_space(1))) const void GlobalPtr;
typedef __attribute__((address_space(3))) void LdsPtr;

template <int TILE, int WAVES, int PRODUCTS, int MODE>
__global__ __launch_bounds__(WAVES *kWave) void product_kernel(MuonCall c, int step, int first_block, int blocks) {
    constexpr int kParts = PRODUCTS == 1 ? 1 : 2;
    constexpr int kWaveRows = 2, kWaveCols = WAVES / kWaveRows;
    constexpr int kRows = TILE / kWaveRows / 16, kCols = TILE / kWaveCols / 16;     // 16 x 16 tiles of a wave
    constexpr int kPanel = TILE * kDepth;                   // halves of a panel
    __shared__ __attribute__((aligned(16))) half_t lds[2][2 * kParts][kPanel];

    // neighbouring tiles on one XCD
    const int b = first_block + int(blockIdx.x), share = blocks / 8, rest = blocks % 8, xcd = b % 8;
    int id = (xcd < rest ? xcd * (share + 1) : rest + xcd * share) + b / 8, which = 0;
    for (;; ++which) {
        const int n = tiles_of(c.t[which], MODE, TILE);
        if (id < n) break;
        id -= n;
    }
    const MuonTensor &t = c.t[which];
    half_t *base = matrices(c, t);
    const Places place(t);
    const int m = t.m, n = t.n;
    int ti, tj;
    if (MODE == kGram || MODE == kSquare) {
        ti = int((sqrtf(8.0f * float(id) + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > id) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
        tj = id - ti * (ti + 1) / 2;
    } else {
        // four tiles of rows at a time
        const int rows = m / TILE, cols = n / TILE, band = id / (4 * cols), first = band * 4;
        const int height = rows - first < 4 ? rows - first : 4;
        ti = first + (id - band * 4 * cols) % height;
        tj = (id - band * 4 * cols) / height;
    }
    const int K = MODE == kGram ? n : m;
    const int64_t ph = MODE == kGram ? place.x(step, 0) : MODE == kSquare ? place.a(0) : place.b(0);
    const int64_t pl = MODE == kGram ? place.x(step, 1) : MODE == kSquare ? place.a(1) : place.b(1);
    const int64_t qh = MODE == kGram ? ph : MODE == kSquare ? ph : place.xt(step, 0);
    const int64_t ql = MODE == kGram ? pl : MODE == kSquare ? pl : place.xt(step, 1);
    const int lane = lane_id(), w = wave_id();

    // A wave's load takes 16 rows of a panel: lane l brings the piece that stands at l.
    const int row = lane >> 2, k8 = piece(row, lane & 3) * 8;
    const int64_t po = int64_t(ti) * TILE * K + int64_t(row) * K + k8, qo = int64_t(tj) * TILE * K + int64_t(row) * K + k8;
    auto fetch = [&](int buffer, int k) {
#pragma unroll
        for (int part = 0; part < 2 * kParts; ++part) {
            const half_t *from = base + (part == 0 ? ph + po : part == 1 ? qh + qo : part == 2 ? pl + po : ql + qo) + k;
#pragma unroll
            for (int q = 0; q < TILE / 16 / WAVES; ++q) {
                const int rows = (q * WAVES + w) * 16;
                __builtin_amdgcn_global_load_lds((GlobalPtr *)(from + int64_t(rows) * K),
                                                 (LdsPtr *)&lds[buffer][part][rows * kDepth], 16, 0, 0);
            }
        }
    };
    Float4 acc[kRows][kCols];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[i][j] = Float4{0.0f, 0.0f, 0.0f, 0.0f};
    const int wr = w / kWaveCols * (kRows * 16), wc = w % kWaveCols * (kCols * 16);
    const int mine = (lane & 15) * kDepth + piece(lane & 15, lane >> 4) * 8;
    auto part_of = [&](int buffer, int part, int at) {
        return *reinterpret_cast<const Half8 *>(&lds[buffer][part][at * kDepth + mine]);
    };
    fetch(0, 0);
    int buffer = 0;
    for (int k = 0; k < K; k += kDepth, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                    // this buffer is there, the other one read
        if (k + kDepth < K) fetch(buffer ^ 1, k + kDepth);
        Half8 qh_[kCols], ql_[kParts == 2 ? kCols : 1];
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            qh_[j] = part_of(buffer, 1, wc + j * 16);
            if (kParts == 2) ql_[j] = part_of(buffer, 3, wc + j * 16);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const Half8 hi = part_of(buffer, 0, wr + i * 16);
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, qh_[j], acc[i][j], 0, 0, 0);
            if (kParts == 2) {
                const Half8 lo = part_of(buffer, 2, wr + i * 16);
#pragma unroll
                for (int j = 0; j < kCols; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, ql_[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, qh_[j], acc[i][j], 0, 0, 0);
                }
            }
        }
    }
    // A lane holds rows 4 (l / 16) to + 3 of column l % 16 of each 16 x 16 tile.
    const int r0 = ti * TILE + wr + (lane >> 4) * 4, c0 = tj * TILE + wc + (lane & 15);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            const int r = r0 + i * 16, q = c0 + j * 16;
            float v[4];
            if (MODE == kGram || MODE == kSquare) {
                // the value times its scale; of a symmetric matrix [q][r] stands for [r][q]
                half_t *th = base + (MODE == kGram ? place.a(0) : place.b(0));
                half_t *tl = base + (MODE == kGram ? place.a(1) : place.b(1));
                const int64_t to = int64_t(q) * m + r;
                if (MODE == kGram) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e] * (1.0f / kScaleX);
                } else {
                    const Half4 ah = *reinterpret_cast<const Half4 *>(base + place.a(0) + to);
                    const Half4 al = *reinterpret_cast<const Half4 *>(base + place.a(1) + to);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = kB * (kScaleB / kScaleX) * (float(ah[e]) + float(al[e])) +
                               kC * (kScaleB / kScaleX / kScaleX) * acc[i][j][e];
                }
                Half4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Split s = split(v[e]);
                    hi[e] = s.hi;
                    lo[e] = s.lo;
                }
                *reinterpret_cast<Half4 *>(th + to) = hi;
                *reinterpret_cast<Half4 *>(tl + to) = lo;
                if (ti != tj) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        th[int64_t(r + e) * m + q] = hi[e];
                        tl[int64_t(r + e) * m + q] = lo[e];
                    }
                }
            } else {
                const int64_t to = int64_t(q) * m + r;      // in X^T
                const Half4 xh = *reinterpret_cast<const Half4 *>(base + place.xt(step, 0) + to);
                const Half4 xl = *reinterpret_cast<const Half4 *>(base + place.xt(step, 1) + to);
#pragma unroll
                for (int e = 0; e < 4; ++e)                 // times kScaleX
                    v[e] = kA * (float(xh[e]) + float(xl[e])) + acc[i][j][e] * (1.0f / kScaleB);
                if (MODE == kApply) {
                    half_t *xr = base + place.x(step + 1, 0), *xrl = base + place.x(step + 1, 1);
                    Half4 hi, lo;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const Split s = split(v[e]);
                        hi[e] = s.hi;
                        lo[e] = s.lo;
                        xr[int64_t(r + e) * n + q] = s.hi;
                        if (kParts == 2) xrl[int64_t(r + e) * n + q] = s.lo;
                    }
                    *reinterpret_cast<Half4 *>(base + place.xt(step + 1, 0) + to) = hi;
                    *reinterpret_cast<Half4 *>(base + place.xt(step + 1, 1) + to) = lo;
                } else {
                    const bool turned = t.rows > t.cols;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int pr = turned ? q : r + e, pc = turned ? r + e : q;
                        if (pr >= t.rows || pc >= t.cols) continue;
                        const int64_t p = pr * t.ld_out + pc;
                        float o = v[e] * (1.0f / kScaleX);
                        if (c.update) {
                            o = (t.master ? t.master[p] : load_typed(t.dtype, t.param, p)) * t.keep - t.scale * o;
                            if (t.master) t.master[p] = o;
                        }
                        store_typed(t.dtype, t.param, p, o);
                    }
                }
            }
        }
}

template <int TILE, int WAVES, int PRODUCTS, int MODE>
hipError_t product(const MuonCall &c, int step, hipStream_t s) {
    int blocks = 0;
    for (int i = 0; i < c.count; ++i) blocks += tiles_of(c.t[i], MODE, TILE);
    return over_blocks(blocks, WAVES * kWave, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL((product_kernel<TILE, WAVES, PRODUCTS, MODE>), dim3(n), dim3(WAVES * kWave), 0, s, c,
                           step, int(first), blocks);
    });
}

template <int TILE, int WAVES, int PRODUCTS> hipError_t steps(const MuonCall &c, hipStream_t s) {
    for (int k = 0; k < c.steps; ++k) {
        hipError_t e = product<TILE, WAVES, PRODUCTS, kGram>(c, k, s);
        if (e == hipSuccess) e = product<TILE, WAVES, 3, kSquare>(c, k, s);
        if (e == hipSuccess)
            e = k + 1 < c.steps ? product<TILE, WAVES, PRODUCTS, kApply>(c, k, s)
                                : product<TILE, WAVES, PRODUCTS, kResult>(c, k, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kSmall = 128, kLarge = 256;

// Large tiles read least, and are taken where there are enough of them for the device.
int tile_of(const MuonCall &c) {
    int64_t tiles = 0;
    for (int i = 0; i < c.count; ++i) {
        const int64_t a = (c.t[i].rows + kLarge - 1) / kLarge, b = (c.t[i].cols + kLarge - 1) / kLarge;
        tiles += a * b;
    }
    return tiles >= 256 ? kLarge : kSmall;
}

}  // namespace

int64_t muon_group(MuonCall &c) {
    const int tile = tile_of(c);
    int64_t at = 0;
    for (int i = 0; i < c.count; ++i) {
        MuonTensor &t = c.t[i];
        const int a = (t.rows + tile - 1) / tile * tile, b = (t.cols + tile - 1) / tile * tile;
        t.m = t.rows <= t.cols ? a : b;
        t.n = t.rows <= t.cols ? b : a;
        t.base = at;
        at += Places(t).all();
    }
    return norms_bytes() + 2 * at;
}

hipError_t launch_muon(const MuonCall &c, hipStream_t s) {
    int most = 0, cuts = 0;
    for (int i = 0; i < c.count; ++i) {
        const int n = norm_blocks(c.t[i]);
        most = n > most ? n : most;
        cuts += (c.t[i].m / kCutTile) * (c.t[i].n / kCutTile);
    }
    hipLaunchKernelGGL(norm_kernel, dim3(most, c.count), dim3(kNormThreads), 0, s, c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = over_blocks(cuts, 256, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL(cut_kernel, dim3(n), dim3(256), 0, s, c, int(first));
    });
    if (e != hipSuccess) return e;
    if (tile_of(c) == kLarge) return c.full ? steps<kLarge, 8, 3>(c, s) : steps<kLarge, 8, 1>(c, s);
    return c.full ? steps<kSmall, 4, 3>(c, s) : steps<kSmall, 4, 1>(c, s);
}

}  // namespace darb
