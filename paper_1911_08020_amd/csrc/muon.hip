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
// is hi hi + hi lo + lo hi.  A result of 16 bits may, where its caller asks for that, take hi hi alone
// for A and for the last product: each element is then off by at most 2^-11 of itself, the result by 1
// to 3 10^-3 of its norm (the steps amplify what happens to small singular values as they do these),
// beside its rounding (2^-8 of an element in bf16, 2^-11 in fp16).  A A is computed from both parts
// then too: A is close to a multiple of the identity when m is well below n, and its one large
// diagonal's rounding would be half of the error.  a X is added from both parts, so that what X has in
// no direction does not grow out of its rounding.
//
// Every product is rows by rows, C[i, j] = sum_k P[i, k] Q[j, k]: A from X, A A from A
// (symmetric), and the last one from b A + c A A and X^T, so each step writes X in both
// orders.  Buffers are padded with zeros to multiples of 32, which the steps keep.  All matrices of a
// call go through one launch per product, the longest sums first.
//
// Bound by the matrix cores: 3 (3 m m n + m m m) operations a step (of fp16 products 3 m m n + 3 m m m),
// on whose random operands a large library product in fp16 reaches 1.4 to 1.5 10^15 a second here
// (2.1 on zeros: it is the power).  Measured on MI355X: 4096 x 9216 in fp32 or 16 bits 7.0 ms
// (1.1 10^15; X's product 1.2, A's 1.1, A A's 1.0), with fp16 products 3.8; the eight matrices of a
// 1500-wide model with its momentum's update, fp32 masters of bf16, 4.4 ms (0.4 of it momentum, norm,
// first X and parameters, at 5 TB/s), without masters 4.4, with fp16 products 2.7; eight bf16 matrices
// of 256 x 1024 180 us, with fp16 products 150 (17 launches of 6 to 14 us: a tile's 32 stages one
// after another).  Equal shares of all stages for each workgroup, cut tiles finished by the last to come,
// took 11.9 ms, 10.4 ms and 377 us: workgroups at unlike places of their sums share nothing in L2.
#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 0x1p15f, kScaleB = 0x1p14f;       // of X and A; of b A + c A A
constexpr int kNormBlocks = 1024;       // at most, a matrix
constexpr int kNormTile = 4096;
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

// Matrices are cut into blocks of 16 rows by kDepth columns (1 KB), row of blocks by row of blocks: a
// wave's load to LDS takes one block as it lies.  In a block, the 16-byte pieces of a row are moved
// so that the rows that a read of LDS takes together use different banks.
__device__ __forceinline__ int piece(int row, int k) { return k ^ (4 - (row >> 2) & 3); }
__device__ __forceinline__ int64_t place_of(int row, int col, int cols) {
    return (int64_t(row >> 4) * (cols / kDepth) + col / kDepth) * (16 * kDepth) + (row & 15) * kDepth +
           piece(row & 15, col % kDepth / 8) * 8 + col % 8;
}

// Before the matrices lie the call itself, which the first launch leaves there (launches that carry
// its 3 KB along cost the host more than their kernels), and the partial sums of the norms.
__host__ __device__ constexpr int64_t call_bytes() { return (int64_t(sizeof(MuonCall)) + 255) / 256 * 256; }
__host__ __device__ constexpr int64_t norms_bytes() { return call_bytes() + int64_t(kMuonTensors) * kNormBlocks * 8; }
__device__ __forceinline__ double *norms(const MuonCall &c, int which) {
    return reinterpret_cast<double *>(static_cast<char *>(c.workspace) + call_bytes()) + which * kNormBlocks;
}

__device__ __forceinline__ half_t *matrices(const MuonCall &c, const MuonTensor &t) {
    return reinterpret_cast<half_t *>(static_cast<char *>(c.workspace) + norms_bytes()) + t.base;
}
__device__ __forceinline__ float load_typed(int type, const void *p, int64_t at) {
    if (type == DARB_F32) return static_cast<const float *>(p)[at];
    if (type == DARB_F16) return float(static_cast<const half_t *>(p)[at]);
    return float(static_cast<const bf16_t *>(p)[at]);
}

// n (1 ... 4) elements from `at` on, and as much of 4 as there is.
template <typename T> __device__ __forceinline__ void load4_as(const T *p, int n, float (&f)[4]) {
    if (n == 4) {
        const Loaded<T, 4> x = load_vec<T, 4>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = i < n ? float(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ void load4(int type, const void *p, int64_t at, int n, float (&f)[4]) {
    if (type == DARB_F32) load4_as(static_cast<const float *>(p) + at, n, f);
    else if (type == DARB_F16) load4_as(static_cast<const half_t *>(p) + at, n, f);
    else load4_as(static_cast<const bf16_t *>(p) + at, n, f);
}
template <typename T> __device__ __forceinline__ void store4_as(T *p, int n, const float (&f)[4]) {
    if (n == 4) {
        store_vec<T, 4>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = T(f[i]);
    }
}
__device__ __forceinline__ void store4(int type, void *p, int64_t at, int n, const float (&f)[4]) {
    if (type == DARB_F32) store4_as(static_cast<float *>(p) + at, n, f);
    else if (type == DARB_F16) store4_as(static_cast<half_t *>(p) + at, n, f);
    else store4_as(static_cast<bf16_t *>(p) + at, n, f);
}

// ---- momentum and norm -----------------------------------------------------------------

__host__ __device__ __forceinline__ int norm_blocks(const MuonTensor &t) {
    const int64_t tiles = (int64_t(t.rows) * t.cols + kNormTile - 1) / kNormTile;
    return int(tiles < kNormBlocks ? tiles : kNormBlocks);
}

__global__ __launch_bounds__(kNormThreads) void norm_kernel(MuonCall c) {
    __shared__ double room[kNormThreads / kWave];
    const int which = int(blockIdx.y);
    if (blockIdx.x == 0 && which == 0)
        for (int i = threadIdx.x; i < int(sizeof(MuonCall) / 4); i += kNormThreads)
            static_cast<uint32_t *>(c.workspace)[i] = reinterpret_cast<const uint32_t *>(&c)[i];
    const MuonTensor &t = c.t[which];
    const int blocks = norm_blocks(t);
    if (int(blockIdx.x) >= blocks) return;
    const float gs = c.grad_scale ? *c.grad_scale : 1.0f;
    const int64_t n = int64_t(t.rows) * t.cols, stride = int64_t(blocks) * kNormThreads * 4;
    const bool dense = t.ld_in == t.cols;
    double sum = 0.0;
#pragma unroll 2
    for (int64_t e = (int64_t(blockIdx.x) * kNormThreads + threadIdx.x) * 4; e < n; e += stride) {
        const int some = n - e < 4 ? int(n - e) : 4;
        float u[4], m[4];
        if (dense) {
            load4(t.gdtype, t.grad, e, some, u);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                u[i] = i < some ? load_typed(t.gdtype, t.grad, (e + i) / t.cols * t.ld_in + (e + i) % t.cols) : 0.0f;
        }
        if (t.momentum) load4(DARB_F32, t.momentum, e, some, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] *= gs;
            if (t.momentum) {
                m[i] = c.mu * m[i] + c.one_mu * u[i];
                u[i] = c.nesterov ? c.mu * m[i] + c.one_mu * u[i] : m[i];
            }
            if (i < some) sum += double(u[i]) * double(u[i]);
        }
        if (t.momentum) store4(DARB_F32, t.momentum, e, some, m);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane_id() == 0) room[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / kWave; ++w) sum += room[w];
        norms(c, which)[blockIdx.x] = sum;
    }
}

// What the workgroups of a launch look for their matrix in.  It travels with the launch: out of the
// call in memory each matrix on the way costs a load that the next one waits for (eight matrices of
// 256 x 1024, fp16 products: 164 us instead of 147).
struct Shares {
    int count;
    int tiles[kMuonTensors];
    uint8_t which[kMuonTensors];
};

// ---- X of the first step ---------------------------------------------------------------

struct Split {
    half_t hi, lo;
};
__device__ __forceinline__ Split split(float scaled) {
    const half_t hi = half_t(scaled);
    return {hi, half_t(scaled - float(hi))};
}

// Padded, in the natural orientation.
__host__ __device__ __forceinline__ int padded_rows(const MuonTensor &t) { return t.rows <= t.cols ? t.m : t.n; }
__host__ __device__ __forceinline__ int padded_cols(const MuonTensor &t) { return t.rows <= t.cols ? t.n : t.m; }

__host__ __device__ __forceinline__ int cut_tiles(const MuonTensor &t) {
    return ((t.m + kCutTile - 1) / kCutTile) * ((t.n + kCutTile - 1) / kCutTile);
}

__global__ __launch_bounds__(256) void cut_kernel(const MuonCall *__restrict__ call, int first_block, Shares shares) {
    const MuonCall &c = *call;
    __shared__ float tile[kCutTile][kCutTile + 1];
    __shared__ double room[256 / kWave];
    int block = first_block + int(blockIdx.x), which = 0;
    for (; which + 1 < shares.count && block >= shares.tiles[which]; ++which) block -= shares.tiles[which];
    const MuonTensor &t = c.t[which];
    const int tid = int(threadIdx.x), R = padded_rows(t), C = padded_cols(t);
    const int across = (C + kCutTile - 1) / kCutTile, r0 = block / across * kCutTile, c0 = block % across * kCutTile;
    const float gs = c.grad_scale ? *c.grad_scale : 1.0f;
    half_t *base = matrices(c, t);
    const Places at(t);
    const bool turned = t.rows > t.cols;                    // X is u^T
    half_t *nh = base + (turned ? at.xt(0, 0) : at.x(0, 0)), *nl = base + (turned ? at.xt(0, 1) : at.x(0, 1));
    half_t *fh = base + (turned ? at.x(0, 0) : at.xt(0, 0)), *fl = base + (turned ? at.x(0, 1) : at.xt(0, 1));
    const int col = tid % 16 * 4;
    float u[kCutTile / 16][4], m[kCutTile / 16][4];
#pragma unroll
    for (int k = 0; k < kCutTile / 16; ++k) {
        const int r = r0 + k * 16 + tid / 16, q = c0 + col, some = r < t.rows ? t.cols - q < 4 ? t.cols - q : 4 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[k][i] = m[k][i] = 0.0f;
        if (some > 0) {
            load4(t.gdtype, t.grad, r * t.ld_in + q, some, u[k]);
            if (t.momentum) load4(DARB_F32, t.momentum, int64_t(r) * t.cols + q, some, m[k]);
        }
    }
    // the norm, beside those loads
    double sum = 0.0;
    for (int i = tid; i < norm_blocks(t); i += 256) sum += norms(c, which)[i];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane_id() == 0) room[wave_id()] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < 256 / kWave; ++w) sum += room[w];
    const double inverse = double(kScaleX) / (sqrt(sum) + c.eps);
#pragma unroll
    for (int k = 0; k < kCutTile / 16; ++k) {
        const int row = k * 16 + tid / 16;
        Half4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = u[k][i] * gs;
            if (t.momentum) x = c.nesterov ? c.mu * m[k][i] + c.one_mu * x : m[k][i];
            x = float(double(x) * inverse);
            tile[row][col + i] = x;
            const Split s = split(x);
            hi[i] = s.hi;
            lo[i] = s.lo;
        }
        if (r0 + row >= R || c0 + col >= C) continue;
        const int64_t to = place_of(r0 + row, c0 + col, C);
        *reinterpret_cast<Half4 *>(nh + to) = hi;
        *reinterpret_cast<Half4 *>(nl + to) = lo;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kCutTile / 16; ++k) {
        const int row = k * 16 + tid / 16;
        Half4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Split s = split(tile[col + i][row]);
            hi[i] = s.hi;
            lo[i] = s.lo;
        }
        if (c0 + row >= C || r0 + col >= R) continue;
        const int64_t to = place_of(c0 + row, r0 + col, R);
        *reinterpret_cast<Half4 *>(fh + to) = hi;
        *reinterpret_cast<Half4 *>(fl + to) = lo;
    }
}

// ---- the products ----------------------------------------------------------------------

enum { kGram, kSquare, kApply, kResult };                   // A; b A + c A A; X; the last X

// Tiles on and below the diagonal, or all of them; the last ones may hang over.
__host__ __device__ __forceinline__ int tiles_of(const MuonTensor &t, int mode, int rows, int cols) {
    const int a = (t.m + rows - 1) / rows;
    return mode == kGram || mode == kSquare ? a * (a + 1) / 2 : a * ((t.n + cols - 1) / cols);
}

// The first and the number of the tiles, of n (below 2^29) of the i-th matrix, that an XCD takes.
__host__ __device__ __forceinline__ int2 share_of(uint32_t n, int xcd, int i) {
    const uint32_t x = uint32_t(xcd + 3 * i) % 8, first = n * x / 8;
    return {int(first), int(n * (x + 1) / 8 - first)};
}

// 16 bytes from each lane's address to LDS, lane after lane from `to` (the same in all lanes).
// In assembly: behind the builtin the compiler lets every read of LDS wait for all such loads,
// those of the other buffer among them (2.1 us a stage of 256 x 256 then).  It has no result in
// registers; `arrived` waits for it.  The load may read M0 only one wait state after it is written,
// which the compiler looks after for the builtin but not inside of assembly: hence the s_nop.  M0
// is listed as written, which a reserved register is warned of.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(const half_t *from, half_t *to) {
    const uint32_t place = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) half_t *)to));
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :: "v"(from), "s"(__builtin_amdgcn_readfirstlane(int(place))) : "memory", "m0");
}
#pragma clang diagnostic pop

// The workgroup's loads to LDS but each wave's last LEFT ones are there, its reads of LDS are done.
template <int LEFT> __device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Lane q of four holds a column's rows 0 ... 3; afterwards row q's columns 0 ... 3.
template <int CTRL> __device__ __forceinline__ uint32_t lane_xor(uint32_t x) { return dpp_all<CTRL>(x); }
__device__ __forceinline__ void turn4(uint32_t (&v)[4]) {
    const int lane = lane_id();
    auto swap = [&](uint32_t &a, uint32_t &b, bool odd, auto other) {
        const uint32_t got = other(odd ? a : b);
        (odd ? a : b) = got;
    };
    const bool one = lane & 1, two = lane & 2;
    auto x1 = [](uint32_t x) { return lane_xor<kDppXor1>(x); };
    auto x2 = [](uint32_t x) { return lane_xor<kDppXor2>(x); };
    swap(v[0], v[1], one, x1);
    swap(v[2], v[3], one, x1);
    swap(v[0], v[2], two, x2);
    swap(v[1], v[3], two, x2);
}

// C tiles of TM x TN by WR x WC waves, BUFS stages of them in LDS or on their way there.
template <int TM, int TN, int WR, int WC, int BUFS, int PRODUCTS, int MODE>
__global__ __launch_bounds__(WR *WC *kWave) void product_kernel(const MuonCall *__restrict__ call, int step,
                                                                int first_block, Shares shares) {
    constexpr int kParts = PRODUCTS == 1 ? 1 : 2, kWaves = WR * WC;
    constexpr int kRows = TM / WR / 16, kCols = TN / WC / 16;                       // 16 x 16 tiles of a wave
    constexpr int kBlocks = (TM + TN) / 16, kBlock = 16 * kDepth;                   // of a stage, P's first
    constexpr bool kTriangle = MODE == kGram || MODE == kSquare;
    constexpr int kLoads = kBlocks / kWaves * kParts;       // of a wave, a stage, at least
    static_assert(!kTriangle || TM == TN, "the diagonal runs through whole tiles");
    static_assert((BUFS - 1) * kLoads < 64, "what s_waitcnt counts");
    __shared__ __attribute__((aligned(16))) half_t lds[BUFS][kParts][kBlocks * kBlock];
    const MuonCall &c = *call;

    // the longest products first; of each matrix a share of neighbouring tiles on one XCD
    const int b = first_block + int(blockIdx.x), xcd = b % 8;
    int id = b / 8, which = -1;
    for (int i = 0; i < shares.count; ++i) {
        const int2 part = share_of(shares.tiles[i], xcd, i);
        if (id < part.y) {
            which = shares.which[i];
            id += part.x;
            break;
        }
        id -= part.y;
    }
    if (which < 0) return;                                  // this XCD's shares are fewer
    const MuonTensor &t = c.t[which];
    half_t *base = matrices(c, t);
    const Places place(t);
    const int m = t.m, n = t.n, K = MODE == kGram ? n : m;
    // four rows of tiles at a time, column by column, and what is on and below the diagonal last
    const int down = (m + TM - 1) / TM, across = kTriangle ? 0 : (n + TN - 1) / TN;
    int ti, tj, top = 0, height;
    for (;; top += 4) {
        height = down - top < 4 ? down - top : 4;
        const int band = kTriangle ? height * top + height * (height + 1) / 2 : height * across;
        if (id < band) break;
        id -= band;
    }
    if (!kTriangle || id < height * top) {
        ti = top + id % height;
        tj = id / height;
    } else {
        id -= height * top;
        ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3;
        tj = top + id - ti * (ti + 1) / 2;
        ti += top;
    }
    const int lane = lane_id(), w = wave_id();
    const int wr = w / WC * (kRows * 16), wc = w % WC * (kCols * 16);
    const int mine = (lane & 15) * kDepth + piece(lane & 15, lane >> 4) * 8;
    auto part_of = [&](int buffer, int part, int at) {
        return *reinterpret_cast<const Half8 *>(&lds[buffer][part][at * kDepth + mine]);
    };
    const int64_t ph = MODE == kGram ? place.x(step, 0) : MODE == kSquare ? place.a(0) : place.b(0);
    const int64_t pl = MODE == kGram ? place.x(step, 1) : MODE == kSquare ? place.a(1) : place.b(1);
    const int64_t qh = kTriangle ? ph : place.xt(step, 0);
    const int64_t ql = kTriangle ? pl : place.xt(step, 1);
    // rows of blocks: behind the last one its own are read again, and not used
    const int plast = m / 16 - 1, qlast = (kTriangle ? m : n) / 16 - 1;
    auto fetch = [&](int buffer, int k) {
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int i = 0; i < (kBlocks + kWaves - 1) / kWaves; ++i) {
                const int at = i * kWaves + w;
                if (kBlocks % kWaves != 0 && at >= kBlocks) break;
                const bool p = at < TM / 16;
                int r = p ? ti * (TM / 16) + at : tj * (TN / 16) + at - TM / 16;
                r = p ? (r < plast ? r : plast) : (r < qlast ? r : qlast);
                const half_t *from = base + (p ? (part ? pl : ph) : (part ? ql : qh)) + int64_t(r) * 16 * K + int64_t(k) * 16;
                load_lds(from + lane * 8, &lds[buffer][part][at * kBlock]);
            }
    };
    Float4 acc[kRows][kCols];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[i][j] = Float4{0.0f, 0.0f, 0.0f, 0.0f};
    // Rows are read two steps ahead, columns a stage: the barrier stands before the last two rows'
    // products, beside which the next stage's first reads run.
    constexpr int kAhead = 2;
    static_assert(kRows >= kAhead, "rows ahead");
    Half8 qh_[kCols], ql_[kCols], hi[kAhead], lo[kAhead];
    auto columns = [&](int buffer) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            qh_[j] = part_of(buffer, 0, TM + wc + j * 16);
            if (kParts == 2) ql_[j] = part_of(buffer, 1, TM + wc + j * 16);
        }
    };
    auto rows = [&](int buffer, int i) {
        hi[i % kAhead] = part_of(buffer, 0, wr + i * 16);
        if (kParts == 2) lo[i % kAhead] = part_of(buffer, 1, wr + i * 16);
    };
    // behind the last stage that one is loaded again, so that the loads on their way stay as many
#pragma unroll
    for (int q = 0; q < BUFS; ++q) fetch(q, q * kDepth < K ? q * kDepth : K - kDepth);
    arrived<(BUFS - 1) * kLoads>();
    columns(0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) rows(0, i);
    int buffer = 0;
    for (int k = 0; k < K; k += kDepth) {
        const int next = buffer + 1 == BUFS ? 0 : buffer + 1;
        Half8 ch[kCols], cl[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) ch[j] = qh_[j], cl[j] = ql_[j];
        Half8 nh[kAhead], nl[kAhead];                       // the next stage's first rows
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const Half8 h = hi[i % kAhead], l = lo[i % kAhead];
            if (i + kAhead < kRows) {
                rows(buffer, i + kAhead);
            } else if (i + kAhead == kRows && k + kDepth < K) {
                arrived<(BUFS - 2) * kLoads>();
                fetch(buffer, k + BUFS * kDepth < K ? k + BUFS * kDepth : K - kDepth);
                columns(next);
#pragma unroll
                for (int r = 0; r < kAhead; ++r) {
                    nh[r] = part_of(next, 0, wr + r * 16);
                    if (kParts == 2) nl[r] = part_of(next, 1, wr + r * 16);
                }
            }
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, ch[j], acc[i][j], 0, 0, 0);
            if (kParts == 2) {
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, cl[j], acc[i][j], 0, 0, 0);
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l, ch[j], acc[i][j], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) hi[i] = nh[i], lo[i] = nl[i];
        buffer = next;
    }
    arrived<0>();                                           // loads to LDS end before the workgroup does
    // A lane holds rows 4 (l / 16) to + 3 of column l % 16 of each 16 x 16 tile, and after turn4
    // columns 4 (l % 16 / 4) to + 3 of row 4 (l / 16) + l % 4.
    const int r0 = ti * TM + wr + (lane >> 4) * 4, c0 = tj * TN + wc + (lane & 15);
    const int r1 = ti * TM + wr + (lane >> 4) * 4 + (lane & 3), c1 = tj * TN + wc + (lane & 12);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            const int r = r0 + i * 16, q = c0 + j * 16, rt = r1 + i * 16, qt = c1 + j * 16;
            // 16 rows or columns at a time are there or not, for all lanes
            if (ti * TM + wr + i * 16 > plast * 16 || tj * TN + wc + j * 16 > qlast * 16) continue;
            float v[4];
            // [q][r ... r + 3] of X^T or a symmetric matrix
            const int64_t to = place_of(q, r, m);
            // both orders of a matrix, hi and lo
            auto write = [&](half_t *th, half_t *tl, half_t *nh, half_t *nl, int ld, bool low) {
                Half4 hi, lo;
                uint32_t both[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Split s = split(v[e]);
                    hi[e] = s.hi;
                    lo[e] = s.lo;
                    both[e] = uint32_t(__builtin_bit_cast(uint16_t, s.hi)) |
                              uint32_t(__builtin_bit_cast(uint16_t, s.lo)) << 16;
                }
                *reinterpret_cast<Half4 *>(th + to) = hi;
                *reinterpret_cast<Half4 *>(tl + to) = lo;
                if (!nh) return;
                turn4(both);
                const int64_t at2 = place_of(rt, qt, ld);
                typedef uint32_t U2 __attribute__((ext_vector_type(2)));
                *reinterpret_cast<U2 *>(nh + at2) = U2{(both[0] & 0xFFFF) | both[1] << 16, (both[2] & 0xFFFF) | both[3] << 16};
                if (low)
                    *reinterpret_cast<U2 *>(nl + at2) =
                        U2{both[0] >> 16 | (both[1] & 0xFFFF0000), both[2] >> 16 | (both[3] & 0xFFFF0000)};
            };
            if (kTriangle) {
                // the value times its scale
                half_t *th = base + (MODE == kGram ? place.a(0) : place.b(0));
                half_t *tl = base + (MODE == kGram ? place.a(1) : place.b(1));
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
                write(th, tl, ti != tj ? th : nullptr, tl, m, true);
            } else {
                const Half4 xh = *reinterpret_cast<const Half4 *>(base + place.xt(step, 0) + to);
                const Half4 xl = *reinterpret_cast<const Half4 *>(base + place.xt(step, 1) + to);
#pragma unroll
                for (int e = 0; e < 4; ++e)             // times kScaleX
                    v[e] = kA * (float(xh[e]) + float(xl[e])) + acc[i][j][e] * (1.0f / kScaleB);
                if (MODE == kApply) {
                    write(base + place.xt(step + 1, 0), base + place.xt(step + 1, 1), base + place.x(step + 1, 0),
                          base + place.x(step + 1, 1), n, kParts == 2);
                } else {
                    const bool turned = t.rows > t.cols;
                    if (!turned) {
                        uint32_t u[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(v[e]);
                        turn4(u);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(u[e]);
                    }
                    const int pr = turned ? q : rt, pc = turned ? r : qt;
                    const int some = pr < t.rows ? t.cols - pc < 4 ? t.cols - pc : 4 : 0;
                    if (some > 0) {
                        const int64_t p = pr * t.ld_out + pc;
                        float o[4];
                        if (c.update) load4(t.master ? int(DARB_F32) : t.dtype, t.master ? t.master : t.param, p, some, o);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] *= 1.0f / kScaleX;
                            if (c.update) v[e] = o[e] * t.keep - t.scale * v[e];
                        }
                        if (c.update && t.master) store4(DARB_F32, t.master, p, some, v);
                        store4(t.dtype, t.param, p, some, v);
                    }
                }
            }
        }
}

// The tiles that a product may go by: rows, columns, and the rate of a compute unit that is full
// of them, of that of the largest.  Measured, us of A, b A + c A A and X:
//   4096 x 9216 fp32       256: 574 277 919   256 x 192: X 795   192: 414 205 985   128: 584 272 838
//                          64: 610 274 1192
//   four of 1500 x 1500, four of 1500 x 6000, fp32 masters
//                          256: 387 134 459   192: 259 157 454   128: 258 124 466
//   eight of 256 x 1024, fp16 products   256: 33 30 28   192: 22 20 19   128: 17 17 15   64: 10 7 10
struct Tile {
    int rows, cols;
    float rate;
};
constexpr Tile kTiles[] = {{256, 256, 1.0f}, {256, 192, 0.9f}, {192, 192, 0.87f}, {128, 128, 0.8f}, {64, 64, 0.5f}};
constexpr int kTileKinds = 5;
constexpr int kUnits = 256;             // compute units

int depth_of(const MuonTensor &t, int mode) { return mode == kGram ? t.n : t.m; }

// How long a product of all matrices takes by tiles of one kind, in stages of the largest: rounds of
// tiles over the compute units, or, where tiles are of unlike lengths, what they come to together and
// half of the shortest.
float cost_of(const MuonCall &c, int mode, const Tile &k) {
    int64_t tiles = 0, all = 0;
    int least = 1 << 30, most = 0;
    for (int i = 0; i < c.count; ++i) {
        const int n = tiles_of(c.t[i], mode, k.rows, k.cols), depth = depth_of(c.t[i], mode);
        tiles += n;
        all += int64_t(n) * depth;
        least = depth < least ? depth : least;
        most = depth > most ? depth : most;
    }
    float rounds = least == most ? float((tiles + kUnits - 1) / kUnits) * most : float(all) / kUnits + 0.5f * least;
    rounds = rounds > most ? rounds : most;
    return rounds * k.rows * k.cols / k.rate;
}

int tile_of(const MuonCall &c, int mode) {
    int best = 0;
    float cost = 0.0f;
    for (int i = 0; i < kTileKinds; ++i) {
        if ((mode == kGram || mode == kSquare) && kTiles[i].rows != kTiles[i].cols) continue;
        const float x = cost_of(c, mode, kTiles[i]);
        if (cost == 0.0f || x < cost) cost = x, best = i;
    }
    return best;
}

template <int TM, int TN, int WR, int WC, int BUFS, int PRODUCTS, int MODE>
hipError_t product(const MuonCall &c, int step, hipStream_t s) {
    Shares shares{};
    shares.count = c.count;
    for (int i = 0; i < c.count; ++i) {
        shares.which[i] = c.order[MODE == kGram][i];
        shares.tiles[i] = tiles_of(c.t[shares.which[i]], MODE, TM, TN);
    }
    int most = 0;
    for (int xcd = 0; xcd < 8; ++xcd) {
        int n = 0;
        for (int i = 0; i < c.count; ++i) n += share_of(shares.tiles[i], xcd, i).y;
        most = n > most ? n : most;
    }
    return over_blocks(8 * int64_t(most), WR * WC * kWave, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL((product_kernel<TM, TN, WR, WC, BUFS, PRODUCTS, MODE>), dim3(n), dim3(WR * WC * kWave), 0, s,
                           static_cast<const MuonCall *>(c.workspace), step, int(first), shares);
    });
}

template <int PRODUCTS, int MODE> hipError_t product(const MuonCall &c, int kind, int step, hipStream_t s) {
    // as many stages as LDS holds beside another workgroup of the smaller tiles
    constexpr bool kOne = PRODUCTS == 1;
    if (kind == 0) return product<256, 256, 2, 4, kOne ? 4 : 2, PRODUCTS, MODE>(c, step, s);
    if constexpr (MODE == kApply || MODE == kResult) {
        if (kind == 1) return product<256, 192, 2, 4, 2, PRODUCTS, MODE>(c, step, s);
    }
    if (kind == 2) return product<192, 192, 2, 4, kOne ? 4 : 3, PRODUCTS, MODE>(c, step, s);
    if (kind == 3) return product<128, 128, 2, 2, kOne ? 4 : 2, PRODUCTS, MODE>(c, step, s);
    return product<64, 64, 2, 2, 4, PRODUCTS, MODE>(c, step, s);
}

template <int PRODUCTS> hipError_t steps(const MuonCall &c, hipStream_t s) {
    auto kind = [&](int mode) { return c.kind[mode] >= 0 ? c.kind[mode] : tile_of(c, mode); };
    const int gram = kind(kGram), square = kind(kSquare), apply = kind(kApply);
    for (int k = 0; k < c.steps; ++k) {
        hipError_t e = product<PRODUCTS, kGram>(c, gram, k, s);
        if (e == hipSuccess) e = product<3, kSquare>(c, square, k, s);
        if (e == hipSuccess)
            e = k + 1 < c.steps ? product<PRODUCTS, kApply>(c, apply, k, s) : product<PRODUCTS, kResult>(c, apply, k, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

static void pad(MuonTensor &t) {
    const int a = (t.rows + kDepth - 1) / kDepth * kDepth, b = (t.cols + kDepth - 1) / kDepth * kDepth;
    t.m = t.rows <= t.cols ? a : b;
    t.n = t.rows <= t.cols ? b : a;
}

int64_t muon_bytes(int64_t rows, int64_t cols) {
    MuonTensor t{};
    t.rows = int32_t(rows), t.cols = int32_t(cols);
    pad(t);
    return 2 * Places(t).all();
}

int64_t muon_group(MuonCall &c) {
    int64_t at = 0;
    for (int i = 0; i < c.count; ++i) {
        MuonTensor &t = c.t[i];
        pad(t);
        t.base = at;
        at += Places(t).all();
    }
    // by length of the products' sums, longest first
    for (int gram = 0; gram < 2; ++gram)
        for (int i = 0; i < c.count; ++i) {
            int j = i;
            const int depth = depth_of(c.t[i], gram ? kGram : kSquare);
            for (; j > 0 && depth_of(c.t[c.order[gram][j - 1]], gram ? kGram : kSquare) < depth; --j)
                c.order[gram][j] = c.order[gram][j - 1];
            c.order[gram][j] = uint8_t(i);
        }
    return norms_bytes() + 2 * at;
}

hipError_t launch_muon(const MuonCall &c, hipStream_t s) {
    int most = 0, cuts = 0;
    Shares shares{};
    shares.count = c.count;
    for (int i = 0; i < c.count; ++i) {
        shares.tiles[i] = cut_tiles(c.t[i]);
        const int n = norm_blocks(c.t[i]);
        most = n > most ? n : most;
        cuts += shares.tiles[i];
    }
    hipLaunchKernelGGL(norm_kernel, dim3(most, c.count), dim3(kNormThreads), 0, s, c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = over_blocks(cuts, 256, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL(cut_kernel, dim3(n), dim3(256), 0, s,
                           static_cast<const MuonCall *>(c.workspace), int(first), shares);
    });
    if (e != hipSuccess) return e;
    return c.full ? steps<3>(c, s) : steps<1>(c, s);
}

}  // namespace darb
