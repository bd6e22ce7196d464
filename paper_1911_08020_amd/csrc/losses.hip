// Losses of policy and preference training over token log probabilities, with their gradients by
// them.
//
//   policy      L_b = -min(r A, clip(r, 1 - e_low, 1 + e_high) A) + c_kl (e^q - 1 - q) - c_h H,
//               r = e^(lp - old), q = ref - lp;  loss = sum_b w_b L_b
//   preference  m_p = beta (s_p - s_{P+p}), s = a sequence's sum of lp - ref,
//               L_p = -(1 - e) log sigma(m_p) - e log sigma(-m_p);  loss = sum_p w_p L_p
//
// Whether a ratio is past its bound is an exact comparison of lp - old, formed in 64 bits, with
// the bound's logarithm; every sum is in 64 bits and in an order that the sizes fix.  A policy
// token is read, its gradient written and its loss added by one thread; a pair's two sequences
// are summed and their gradients filled in by one workgroup.  The workgroups' sums are added by a
// second launch of one workgroup (the first one does it where there is only that).
//
// Memory-bound for many tokens, latency-bound for few.  Kernel times, with sums launch: policy 4.1 us
// for 700 tokens (one launch) and 8.1 + 3.3 us for 1 M (24 MB from the Infinity Cache), preference
// 6.1 + 2.1 us for 64 padded pairs' 512 tokens and 8.3 + 3.0 us for 1500 packed pairs of 2.1 M tokens.
#include "darb_internal.h"
#include "exp_of.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr int kThreads = 256;
constexpr int kBig = 1024;              // threads of a workgroup that is alone
constexpr int kV = 4;
constexpr int kTile = kThreads * kV;     // policy tokens of a workgroup (16 a thread: 12.5 us for 1 M, not 8.0)
// Tokens that one workgroup takes by itself, the whole call: 8192 6.6 us (two launches 9.9), 16384
// 9.3 (9.5), 32768 15.2 (9.9).
constexpr int kAlone = 8192;

// The workgroup's sums of each thread's x, in thread 0 (`room`: a double a wave for each).
template <int THREADS, int N> __device__ __forceinline__ void block_sums(double (&x)[N], double (&room)[N][THREADS / kWave]) {
    constexpr int kWaves = THREADS / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) x[i] += __shfl_xor(x[i], d);
        if (lane_id() == 0) room[i][wave_id()] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = room[i][threadIdx.x % kWaves];
#pragma unroll
        for (int d = 1; d < kWaves; d <<= 1) x[i] += __shfl_xor(x[i], d);
    }
}

// ---- policy ----------------------------------------------------------------------------

struct Sums {
    double loss = 0.0, kl = 0.0, cut = 0.0;
};

// e^q - 1 - q without its cancellation near 0, and e^q - 1.
__device__ __forceinline__ float excess(float q, float &grown) {
    float p = 1.0f / 362880.0f;
    p = p * q + 1.0f / 40320.0f;
    p = p * q + 1.0f / 5040.0f;
    p = p * q + 1.0f / 720.0f;
    p = p * q + 1.0f / 120.0f;
    p = p * q + 1.0f / 24.0f;
    p = p * q + 1.0f / 6.0f;
    p = p * q + 0.5f;
    p = p * q * q;
    const float e = exp_of(q) - 1.0f;
    const bool near = fabsf(q) < 0.5f;
    grown = near ? p + q : e;
    return near ? p : e - q;
}

struct PolicyToken {
    float lp, old, A, w, ref, h;
};

__device__ __forceinline__ float policy_token(const PolicyCall &c, const PolicyToken &t, Sums &s) {
    if (t.w == 0.0f) return 0.0f;       // whatever stands there
    const double d = double(t.lp) - double(t.old);
    // a finite ratio times 0, where fp32 holds the ratio as infinite too
    const float ra = t.A == 0.0f && isfinite(d) ? 0.0f : exp_of(float(d)) * t.A;
    float loss = -ra, grad = -ra;
    if (t.A > 0.0f && d > c.log_high) {
        loss = -(c.high * t.A);
        grad = 0.0f;
        s.cut += double(t.w);
    } else if (t.A < 0.0f && d < c.log_low) {
        loss = -(c.low * t.A);
        grad = 0.0f;
        s.cut += double(t.w);
    }
    if (c.ref) {
        const float q = float(double(t.ref) - double(t.lp));
        float grown;
        const float k = excess(q, grown);
        s.kl += double(t.w) * double(k);
        if (c.kl_coef != 0.0f) {        // 0: kl is only summed, whatever it comes to
            loss += c.kl_coef * k;
            grad -= c.kl_coef * grown;
        }
    }
    if (c.entropy) loss -= c.entropy_coef * t.h;
    s.loss += double(t.w) * double(loss);
    return grad * t.w;
}

__device__ __forceinline__ void load4(const float *p, int64_t at, int n, float none, float (&f)[kV]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < kV; ++i) f[i] = none;
    } else if (n == kV) {
        const Loaded<float, kV> x = load_vec<float, kV>(p + at);
#pragma unroll
        for (int i = 0; i < kV; ++i) f[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) f[i] = i < n ? p[at + i] : 0.0f;
    }
}

__device__ __forceinline__ void store4(float *p, int64_t at, int n, const float (&f)[kV]) {
    if (n == kV) {
        store_vec<float, kV>(p + at, f);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (i < n) p[at + i] = f[i];
    }
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void policy_kernel(PolicyCall c, int64_t first_block, int64_t blocks, int64_t tile) {
    __shared__ double room[3][THREADS / kWave];
    Sums s;
    const int64_t block = first_block + blockIdx.x, end = (block + 1) * tile < c.B ? (block + 1) * tile : c.B;
    for (int64_t at = block * tile + int64_t(threadIdx.x) * kV; at < end; at += THREADS * kV) {
        const int n = end - at >= kV ? kV : int(end - at);
        float lp[kV], old[kV], A[kV], w[kV], ref[kV], h[kV], g[kV], gh[kV];
        load4(c.lp, at, n, 0.0f, lp);
        load4(c.old, at, n, 0.0f, old);
        load4(c.advantage, at, n, 0.0f, A);
        load4(c.weight, at, n, c.even, w);
        load4(c.ref, at, n, 0.0f, ref);
        load4(c.entropy, at, n, 0.0f, h);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            g[i] = i < n ? policy_token(c, {lp[i], old[i], A[i], w[i], ref[i], h[i]}, s) : 0.0f;
            gh[i] = -(c.entropy_coef * w[i]);
        }
        store4(c.grad, at, n, g);
        if (c.grad_entropy) store4(c.grad_entropy, at, n, gh);
    }
    double x[3] = {s.loss, s.kl, s.cut};
    block_sums<THREADS>(x, room);
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        if (blocks == 1) c.stats[q] = float(x[q]);
        else c.partial[q * blocks + block] = x[q];
    }
}

__global__ __launch_bounds__(kThreads) void policy_sum_kernel(const double *partial, int64_t blocks, float *stats) {
    __shared__ double room[3][kThreads / kWave];
    double x[3] = {};
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < blocks; i += kThreads) {
#pragma unroll
        for (int q = 0; q < 3; ++q) x[q] += partial[q * blocks + i];
    }
    block_sums<kThreads>(x, room);
    if (threadIdx.x == 0) {
#pragma unroll
        for (int q = 0; q < 3; ++q) stats[q] = float(x[q]);
    }
}

int64_t policy_blocks(int64_t B) { return B <= kAlone ? 1 : (B + kTile - 1) / kTile; }

// ---- preferences -----------------------------------------------------------------------

__device__ __forceinline__ float pair_loss(const PreferenceCall &c, float m, float w) {
    if (w == 0.0f) return 0.0f;
    const float l = log1pf(expf(-fabsf(m)));
    const float down = fmaxf(-m, 0.0f) + l, up = fmaxf(m, 0.0f) + l;    // - log sigma(m), (-m)
    return w * ((1.0f - c.smoothing) * down + (c.smoothing != 0.0f ? c.smoothing * up : 0.0f));
}

// Pair p's sequences are p and P + p.  Strided: token t of sequence s at t * 2P + s; packed: the
// tokens starts[s] to starts[s + 1].  PAIRS pairs a workgroup (strided ones side by side).
template <int THREADS, int PAIRS>
__global__ __launch_bounds__(THREADS) void preference_kernel(PreferenceCall c, int64_t first_block, bool alone) {
    __shared__ double room[2 * PAIRS][THREADS / PAIRS / 2];
    __shared__ float coef[2 * PAIRS];
    constexpr int kTeam = THREADS / (2 * PAIRS);            // threads of a sequence
    constexpr int kLine = kTeam < kWave ? kTeam : kWave;
    const int64_t block = first_block + blockIdx.x, S = 2 * c.P;
    const int q = int(threadIdx.x) % (2 * PAIRS), team = int(threadIdx.x) / (2 * PAIRS);
    // strided: lanes lie side by side over the sequences; packed: over the tokens
    const int which = c.starts ? int(threadIdx.x) / kTeam : q, at = c.starts ? int(threadIdx.x) % kTeam : team;
    const int64_t pair = block * PAIRS + which % PAIRS, s = which < PAIRS ? pair : c.P + pair;
    int64_t from = 0, count = 0, stride = 1, head = 0, tail = 0;
    if (c.starts) {
        head = c.starts[0];
        tail = c.starts[S];
    }
    if (pair < c.P) {
        if (c.starts) {
            int64_t a = c.starts[s], b = c.starts[s + 1];
            a = a < 0 ? 0 : a > c.B ? c.B : a;              // never outside the tokens
            b = b < a ? a : b > c.B ? c.B : b;
            from = a;
            count = b - a;
        } else {
            from = s;
            count = c.L;
            stride = S;
        }
    }
    double sum = 0.0;
    if (c.starts) {
#pragma unroll 2
        for (int64_t t = int64_t(at) * kV; t < count; t += kTeam * kV) {
            const int n = count - t < kV ? int(count - t) : kV;
            float lp[kV], ref[kV];
            load4(c.lp, from + t, n, 0.0f, lp);
            load4(c.ref, from + t, n, 0.0f, ref);
#pragma unroll
            for (int i = 0; i < kV; ++i) sum += double(lp[i]) - double(ref[i]);
        }
    } else {
#pragma unroll 8
        for (int64_t t = at; t < count; t += kTeam) {
            const int64_t e = from + t * stride;
            sum += double(c.lp[e]) - (c.ref ? double(c.ref[e]) : 0.0);
        }
    }
    // each sequence's parts by neighbouring lanes, whichever way they were read
    room[which][at] = sum;
    __syncthreads();
    sum = room[threadIdx.x / kTeam][threadIdx.x % kTeam];
#pragma unroll
    for (int d = 1; d < kLine; d <<= 1) sum += __shfl_xor(sum, d);
    __syncthreads();
    if (threadIdx.x % kLine == 0) room[threadIdx.x / kTeam][threadIdx.x % kTeam / kLine] = sum;
    __syncthreads();
    if (threadIdx.x < PAIRS && block * PAIRS + threadIdx.x < c.P) {
        const int j = int(threadIdx.x);
        const int64_t p = block * PAIRS + j;
        double good = 0.0, bad = 0.0;
#pragma unroll
        for (int i = 0; i < kTeam / kLine; ++i) {
            good += room[j][i];
            bad += room[PAIRS + j][i];
        }
        const float m = float(double(c.beta) * (good - bad)), w = c.weight ? c.weight[p] : c.even;
        const float e = expf(-fabsf(m));
        const float below = (m >= 0.0f ? e : 1.0f) / (1.0f + e);        // sigma(-m)
        const float d = w == 0.0f ? 0.0f : (c.smoothing - below) * (c.beta * w);
        c.margin[p] = m;
        coef[j] = d;
        coef[PAIRS + j] = -d;
    }
    __syncthreads();
    if (pair < c.P) {
        const float d = coef[which];
        if (c.starts) {
            const float all[kV] = {d, d, d, d};
            for (int64_t t = int64_t(at) * kV; t < count; t += kTeam * kV)
                store4(c.grad, from + t, count - t < kV ? int(count - t) : kV, all);
        } else {
            for (int64_t t = at; t < count; t += kTeam) c.grad[from + t * stride] = d;
        }
    }
    if (c.starts) {
        // tokens of no sequence have no gradient: each workgroup clears a share
        head = head < 0 ? 0 : head > c.B ? c.B : head;
        tail = tail < head ? head : tail > c.B ? c.B : tail;
        const int64_t none = head + c.B - tail, all = (c.P + PAIRS - 1) / PAIRS;
        for (int64_t i = block * THREADS + threadIdx.x; i < none; i += all * THREADS)
            c.grad[i < head ? i : tail + (i - head)] = 0.0f;
    }
    if (alone) {
        __syncthreads();
        if (threadIdx.x == 0) {
            double x = 0.0;
            for (int64_t p = 0; p < c.P; ++p) x += double(pair_loss(c, c.margin[p], c.weight ? c.weight[p] : c.even));
            *c.loss = float(x);
        }
    }
}

__global__ __launch_bounds__(kBig) void preference_sum_kernel(PreferenceCall c) {
    __shared__ double room[1][kBig / kWave];
    double x[1] = {0.0};
    for (int64_t p = threadIdx.x; p < c.P; p += kBig)
        x[0] += double(pair_loss(c, c.margin[p], c.weight ? c.weight[p] : c.even));
    block_sums<kBig>(x, room);
    if (threadIdx.x == 0) *c.loss = float(x[0]);
}

}  // namespace

int64_t policy_workspace_bytes(int64_t B) {
    const int64_t blocks = policy_blocks(B);
    return blocks == 1 ? 0 : (24 * blocks + 255) / 256 * 256;
}

hipError_t launch_policy(PolicyCall c, hipStream_t s) {
    const int64_t blocks = policy_blocks(c.B);
    if (blocks == 1) {
        hipLaunchKernelGGL((policy_kernel<kBig>), dim3(1), dim3(kBig), 0, s, c, 0, 1, int64_t(kAlone));
        return hipGetLastError();
    }
    const hipError_t e = over_blocks(blocks, kThreads, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL((policy_kernel<kThreads>), dim3(n), dim3(kThreads), 0, s, c, first, blocks, int64_t(kTile));
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(kThreads), 0, s, c.partial, blocks, c.stats);
    return hipGetLastError();
}

hipError_t launch_preference(const PreferenceCall &c, hipStream_t s) {
    hipError_t e;
    bool alone = false;
    if (c.starts) {
        alone = c.P == 1;
        e = over_blocks(c.P, kThreads, [&](int64_t first, unsigned n) {
            hipLaunchKernelGGL((preference_kernel<kThreads, 1>), dim3(n), dim3(kThreads), 0, s, c, first, alone);
        });
    } else {
        constexpr int kPairs = 4;
        const int64_t blocks = (c.P + kPairs - 1) / kPairs;
        alone = blocks == 1;
        e = over_blocks(blocks, kThreads, [&](int64_t first, unsigned n) {
            hipLaunchKernelGGL((preference_kernel<kThreads, kPairs>), dim3(n), dim3(kThreads), 0, s, c, first, alone);
        });
    }
    if (e != hipSuccess || alone) return e;
    hipLaunchKernelGGL(preference_sum_kernel, dim3(1), dim3(kBig), 0, s, c);
    return hipGetLastError();
}

}  // namespace darb
