// One AdamW step (decoupled weight decay) over many tensors in one launch, with states in 32
// bits or in 8.
//
//   m = m b1 + g (1 - b1),  v = v b2 + g g (1 - b2)
//   p = p (1 - lr decay) - (m / (sqrt(v) / sqrt(1 - b2^t) + eps)) (lr / (1 - b1^t))
//
// Every operation is one correctly rounded fp32 operation in this order (no contraction), so
// the states' 8-bit codes, an integer decision taken from floating point, are defined exactly.
//
// States in 8 bits: blocks of 256 elements share an fp32 scale, the block's greatest magnitude
// a.  With q = |x| / a in [0, 1], a code is the leading bits of the fp32 number q: for m a sign,
// 4 bits of exponent and 3 of mantissa, for v (never negative) 4 and 4, the greatest code
// standing for 1.  Rounding is random: bits below the kept ones are filled by adding uniformly
// random ones, so that the expected value is q.  Rounding to nearest would freeze the averages:
// with b2 = 0.999 a step changes v by about a thousandth, far less than half a code.  m below
// the lowest code becomes 0; v that is not 0 keeps at least the lowest code, so that a step
// never divides by eps alone.  The random bits are a hash of the element's number, the tensor's
// and the step's, the caller's seed among it: the same inputs give the same codes.
//
// Memory-bound: 28 bytes an fp32 element with 32-bit states, 16 with 8-bit ones.  Measured on
// MI355X: 4 M fp32 elements in 14 tensors 19 us (5.9 TB/s, out of the Infinity Cache); 64 M fp16
// ones with fp32 masters and gradients and 8-bit states 225 us (5.1 TB/s), the export of their
// moments 150 (4.3 TB/s, four fifths of it stores).
#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

#pragma clang fp contract(off)

namespace darb {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 4096;             // elements of a workgroup: 16 a thread
constexpr int kV = 4;                   // elements of a thread at a time
constexpr int kRounds = kTile / (kThreads * kV);
static_assert(kAdamBlock == kWave * kV, "a wave takes one block at a time");

struct Scalars {
    float b1, one_b1, b2, one_b2, rs, eps, step;
    double lr;
    const float *grad_scale;
    uint32_t seed;
};

struct Grads {
    const void *p[kAdamGrads];
    uint32_t type[(kAdamGrads + 15) / 16];          // 2 bits each
};

// n of the kV elements at p (all of them where n == kV), the others 0.
template <typename T> __device__ __forceinline__ void load_some(const T *p, int n, float (&f)[kV]) {
    if (n == kV) {
        const Loaded<T, kV> x = load_vec<T, kV>(p);
#pragma unroll
        for (int i = 0; i < kV; ++i) f[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) f[i] = i < n ? float(p[i]) : 0.0f;
    }
}

template <bool STREAM = false, typename T> __device__ __forceinline__ void store_some(T *p, int n, const float (&f)[kV]) {
    if (n == kV) {
        store_vec<T, kV, STREAM>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (i < n) p[i] = T(f[i]);
    }
}

__device__ __forceinline__ void load_typed(int type, const void *p, int64_t at, int n, float (&f)[kV]) {
    if (type == DARB_F32) load_some(static_cast<const float *>(p) + at, n, f);
    else if (type == DARB_F16) load_some(static_cast<const half_t *>(p) + at, n, f);
    else load_some(static_cast<const bf16_t *>(p) + at, n, f);
}

__device__ __forceinline__ void store_typed(int type, void *p, int64_t at, int n, const float (&f)[kV]) {
    if (type == DARB_F32) store_some(static_cast<float *>(p) + at, n, f);
    else if (type == DARB_F16) store_some(static_cast<half_t *>(p) + at, n, f);
    else store_some(static_cast<bf16_t *>(p) + at, n, f);
}

typedef uint32_t u32_any __attribute__((aligned(1)));

__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int n) {
    if (n == kV) return *reinterpret_cast<const u32_any *>(p);
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < kV; ++i)
        if (i < n) c |= uint32_t(p[i]) << (8 * i);
    return c;
}

__device__ __forceinline__ void store_codes(uint8_t *p, int n, uint32_t c) {
    if (n == kV) {
        *reinterpret_cast<u32_any *>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (i < n) p[i] = uint8_t(c >> (8 * i));
    }
}

// ---- 8-bit codes -----------------------------------------------------------------------

constexpr int kShiftM = 20, kLowM = 889, kTopM = 127;     // 1.0 is 1016 << 20
constexpr int kShiftV = 19, kLowV = 1777, kTopV = 255;    // 1.0 is 2032 << 19

__device__ __forceinline__ float value_m(uint32_t code, float scale) {
    const uint32_t c = code & kTopM;
    const float x = (c ? __uint_as_float((c + kLowM) << kShiftM) : 0.0f) * scale;
    return code > kTopM ? -x : x;
}
__device__ __forceinline__ float value_v(uint32_t code, float scale) {
    return (code ? __uint_as_float((code + kLowV) << kShiftV) : 0.0f) * scale;
}

// 32 mixed bits of a counter.
__device__ __forceinline__ uint32_t random_bits(uint32_t x) {
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0xB504F333u;
    return x ^ (x >> 16);
}

// The block's scale and its inverse from the bits of the greatest magnitude: none below 2^-120
// (the inverse could overflow; all codes are 0), NaN where a magnitude is not finite.
__device__ __forceinline__ float scale_of(uint32_t bits, float &inverse) {
    const float a = __uint_as_float(bits);
    if (bits >= 0x7F800000u) {
        inverse = 0.0f;
        return __builtin_nanf("");
    }
    inverse = a < 0x1p-120f ? 0.0f : 1.0f / a;
    return a < 0x1p-120f ? 0.0f : a;
}

__device__ __forceinline__ uint32_t code_m(float x, float inverse, uint32_t random) {
    if (inverse == 0.0f) return 0;
    const int c = int((__float_as_uint(fabsf(x) * inverse) + (random << 4)) >> kShiftM) - kLowM;
    if (c <= 0) return 0;
    return uint32_t(c > kTopM ? kTopM : c) | (x < 0.0f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t code_v(float x, float inverse, uint32_t random) {
    if (inverse == 0.0f || !(x > 0.0f)) return 0;
    const int c = int((__float_as_uint(x * inverse) + (random << 3)) >> kShiftV) - kLowV;
    return uint32_t(c < 1 ? 1 : c > kTopV ? kTopV : c);
}

// ---- the step --------------------------------------------------------------------------

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamTensor *__restrict__ tensors,
                                                         const AdamTile *__restrict__ tiles,
                                                         int first_tensor, Scalars k, Grads grads) {
    const AdamTile tile = tiles[blockIdx.x];
    const AdamTensor t = tensors[tile.tensor];
    const int local = int(tile.tensor) - first_tensor;
    const void *gp = grads.p[local];
    if (!gp) return;                                 // no gradient: the tensor stays as it is
    const int gtype = (grads.type[local / 16] >> (local % 16 * 2)) & 3;
    const float gs = k.grad_scale ? *k.grad_scale : 1.0f;
    const float keep = float(1.0 - k.lr * t.decay);
    const int w = wave_id(), lane = lane_id();
    const int64_t first = int64_t(tile.index) * kTile;
    const uint32_t key = tile.tensor * 0xBB67AE85u + k.seed;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t block = first / kAdamBlock + r * (kThreads / kWave) + w;
        const int64_t at = block * kAdamBlock + lane * kV;
        if (block * kAdamBlock >= t.n) break;        // whole waves
        const int n = t.n - at >= kV ? kV : t.n - at > 0 ? int(t.n - at) : 0;
        float p[kV], g[kV], m[kV], v[kV];
        if (t.master) load_some(t.master + at, n, p);
        else load_typed(t.dtype, t.param, at, n, p);
        load_typed(gtype, gp, at, n, g);
        if (BITS == 32) {
            load_some(static_cast<const float *>(t.m) + at, n, m);
            load_some(static_cast<const float *>(t.v) + at, n, v);
        } else {
            const uint32_t cm = load_codes(static_cast<const uint8_t *>(t.m) + at, n);
            const uint32_t cv = load_codes(static_cast<const uint8_t *>(t.v) + at, n);
            const float sm = t.m_scale[block], sv = t.v_scale[block];
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                m[i] = value_m((cm >> (8 * i)) & 255, sm);
                v[i] = value_v((cv >> (8 * i)) & 255, sv);
            }
        }
        uint32_t am = 0, av = 0;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float x = g[i] * gs;
            m[i] = m[i] * k.b1 + x * k.one_b1;
            v[i] = v[i] * k.b2 + (x * x) * k.one_b2;
            const float d = __builtin_sqrtf(v[i]) * k.rs + k.eps;
            p[i] = p[i] * keep - __fdiv_rn(m[i], d) * k.step;
            if (i < n) {
                const uint32_t bm = __float_as_uint(fabsf(m[i])), bv = __float_as_uint(fabsf(v[i]));
                am = bm > am ? bm : am;
                av = bv > av ? bv : av;
            }
        }
        if (t.master) store_some(t.master + at, n, p);
        store_typed(t.dtype, t.param, at, n, p);
        if (BITS == 32) {
            store_some(static_cast<float *>(t.m) + at, n, m);
            store_some(static_cast<float *>(t.v) + at, n, v);
        } else {
            float im, iv;
            const float sm = scale_of(wave_max_u32(am), im), sv = scale_of(wave_max_u32(av), iv);
            uint32_t cm = 0, cv = 0;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const uint32_t h = random_bits(uint32_t(at + i) + key);
                cm |= code_m(m[i], im, h & 0xFFFFu) << (8 * i);
                cv |= code_v(v[i], iv, h >> 16) << (8 * i);
            }
            store_codes(static_cast<uint8_t *>(t.m) + at, n, cm);
            store_codes(static_cast<uint8_t *>(t.v) + at, n, cv);
            if (lane == 0) {
                t.m_scale[block] = sm;
                t.v_scale[block] = sv;
            }
        }
    }
}

struct Moments {
    float *m[kAdamGrads / 2], *v[kAdamGrads / 2];
};

template <int BITS>
__global__ __launch_bounds__(kThreads) void moments_kernel(const AdamTensor *__restrict__ tensors,
                                                           const AdamTile *__restrict__ tiles,
                                                           int first_tensor, Moments out) {
    const AdamTile tile = tiles[blockIdx.x];
    const AdamTensor t = tensors[tile.tensor];
    float *om = out.m[tile.tensor - first_tensor], *ov = out.v[tile.tensor - first_tensor];
    const int w = wave_id(), lane = lane_id();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t block = int64_t(tile.index) * (kTile / kAdamBlock) + r * (kThreads / kWave) + w;
        const int64_t at = block * kAdamBlock + lane * kV;
        if (block * kAdamBlock >= t.n) break;
        const int n = t.n - at >= kV ? kV : t.n - at > 0 ? int(t.n - at) : 0;
        float m[kV], v[kV];
        if (BITS == 32) {
            load_some(static_cast<const float *>(t.m) + at, n, m);
            load_some(static_cast<const float *>(t.v) + at, n, v);
        } else {
            const uint32_t cm = load_codes(static_cast<const uint8_t *>(t.m) + at, n);
            const uint32_t cv = load_codes(static_cast<const uint8_t *>(t.v) + at, n);
            const float sm = t.m_scale[block], sv = t.v_scale[block];
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                m[i] = value_m((cm >> (8 * i)) & 255, sm);
                v[i] = value_v((cv >> (8 * i)) & 255, sv);
            }
        }
        // past the caches, which they would only sweep: 168 -> 152 us for 64 M elements
        if (om) store_some<true>(om + at, n, m);
        if (ov) store_some<true>(ov + at, n, v);
    }
}

}  // namespace

int64_t adam_tile_elements() { return kTile; }

hipError_t launch_adamw(int bits, const AdamTensor *tensors, const AdamTile *tiles, int64_t ntiles,
                        int first_tensor, int count, const void *const *grads, const int *types,
                        const AdamScalars &c, hipStream_t s) {
    if (ntiles == 0) return hipSuccess;
    const Scalars k{float(c.beta1), float(1.0 - c.beta1), float(c.beta2), float(1.0 - c.beta2),
                    float(1.0 / __builtin_sqrt(1.0 - __builtin_pow(c.beta2, double(c.step)))),
                    float(c.eps),
                    float(c.lr / (1.0 - __builtin_pow(c.beta1, double(c.step)))), c.lr,
                    c.grad_scale, c.seed};
    Grads g{};
    for (int i = 0; i < count; ++i) {
        if (!grads[i]) continue;                     // its type may be anything
        g.p[i] = grads[i];
        g.type[i / 16] |= uint32_t(types[i]) << (i % 16 * 2);
    }
    if (bits == 32)
        hipLaunchKernelGGL((adamw_kernel<32>), dim3(unsigned(ntiles)), dim3(kThreads), 0, s,
                           tensors, tiles, first_tensor, k, g);
    else
        hipLaunchKernelGGL((adamw_kernel<8>), dim3(unsigned(ntiles)), dim3(kThreads), 0, s,
                           tensors, tiles, first_tensor, k, g);
    return hipGetLastError();
}

hipError_t launch_moments(int bits, const AdamTensor *tensors, const AdamTile *tiles,
                          int64_t ntiles, int first_tensor, int count, float *const *m,
                          float *const *v, hipStream_t s) {
    if (ntiles == 0) return hipSuccess;
    Moments o{};
    for (int i = 0; i < count; ++i) {
        o.m[i] = m ? m[i] : nullptr;
        o.v[i] = v ? v[i] : nullptr;
    }
    if (bits == 32)
        hipLaunchKernelGGL((moments_kernel<32>), dim3(unsigned(ntiles)), dim3(kThreads), 0, s,
                           tensors, tiles, first_tensor, o);
    else
        hipLaunchKernelGGL((moments_kernel<8>), dim3(unsigned(ntiles)), dim3(kThreads), 0, s,
                           tensors, tiles, first_tensor, o);
    return hipGetLastError();
}

}  // namespace darb
