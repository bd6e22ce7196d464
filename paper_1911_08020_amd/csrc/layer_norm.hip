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
// and a second launch adds them in a fixed order.
#include <type_traits>

#include "darb_internal.h"
#include "float_io.h"
#include "wave.h"

namespace darb {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxWaves = kMaxThreads / kWave;
constexpr int kAnyThreads = 256;

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
};

template <typename T>
__device__ __forceinline__ float weight_at(const Args &a, const void *w, int64_t h) {
    return a.w_f32 ? static_cast<const float *>(w)[h] : float(static_cast<const T *>(w)[h]);
}

// The workgroup's sum of s[0 .. N), each in every thread; scratch: N * kMaxWaves floats.
template <int N> __device__ __forceinline__ void block_sum(float (&s)[N], float *scratch) {
    const int waves = blockDim.x / kWave, w = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if (waves == 1) return;
    __syncthreads();                                 // the scratch's last use
    if (lane_id() == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) scratch[i * kMaxWaves + w] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = 0.0f;
        for (int k = 0; k < waves; ++k) s[i] += scratch[i * kMaxWaves + k];
    }
}

// ---- any strides and lengths: a workgroup per column, one element at a time ------------

template <typename T>
__global__ __launch_bounds__(kAnyThreads) void any_norm_kernel(Args a) {
    __shared__ float scratch[kMaxWaves];
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const T *x = static_cast<const T *>(a.x.p) + b * a.x.token;
        T *y = static_cast<T *>(a.y.p) + b * a.y.token;
        float s[1] = {0.0f};
        for (int64_t h = threadIdx.x; h < a.H; h += kAnyThreads) s[0] += float(x[h * a.x.feature]);
        block_sum(s, scratch);
        const float mean = s[0] / float(a.H);
        s[0] = 0.0f;
        for (int64_t h = threadIdx.x; h < a.H; h += kAnyThreads) {
            const float d = float(x[h * a.x.feature]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        block_sum(s, scratch);
        const float rstd = 1.0f / sqrtf(s[0] / float(a.H) + a.eps);
        for (int64_t h = threadIdx.x; h < a.H; h += kAnyThreads) {
            float v = (float(x[h * a.x.feature]) - mean) * rstd;
            if (a.w) v *= weight_at<T>(a, a.w, h);
            if (a.b) v += weight_at<T>(a, a.b, h);
            y[h * a.y.feature] = T(v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[b] = mean;
            if (a.rstd) a.rstd[b] = rstd;
        }
    }
}

// The workgroup's columns' dw and db go to its row of the partial sums, element by element.
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void any_norm_grad_kernel(Args a) {
    __shared__ float scratch[2 * kMaxWaves];
    float *dw = a.dw ? a.dw + blockIdx.x * a.H : nullptr;
    float *db = a.db ? a.db + blockIdx.x * a.H : nullptr;
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const T *x = static_cast<const T *>(a.x.p) + b * a.x.token;
        const T *dy = static_cast<const T *>(a.dy.p) + b * a.dy.token;
        T *dx = static_cast<T *>(a.y.p) + b * a.y.token;
        const float mean = a.mean[b], rstd = a.rstd[b];
        const bool first = b == blockIdx.x;
        float s[2] = {0.0f, 0.0f};
        for (int64_t h = threadIdx.x; h < a.H; h += kAnyThreads) {
            const float g = float(dy[h * a.dy.feature]);
            const float xh = (float(x[h * a.x.feature]) - mean) * rstd;
            const float v = a.w ? g * weight_at<T>(a, a.w, h) : g;
            s[0] += v;
            s[1] = fmaf(v, xh, s[1]);
            if (dw) dw[h] = first ? g * xh : fmaf(g, xh, dw[h]);
            if (db) db[h] = first ? g : db[h] + g;
        }
        if (!a.y.p) continue;
        block_sum(s, scratch);
        const float m0 = s[0] / float(a.H), m1 = s[1] / float(a.H);
        for (int64_t h = threadIdx.x; h < a.H; h += kAnyThreads) {
            const float g = float(dy[h * a.dy.feature]);
            const float xh = (float(x[h * a.x.feature]) - mean) * rstd;
            const float v = a.w ? g * weight_at<T>(a, a.w, h) : g;
            dx[h * a.y.feature] = T(rstd * (v - m0 - xh * m1));
        }
        __syncthreads();
    }
}

// ---- the partial sums of dw and db -----------------------------------------------------

constexpr int kSumFeatures = 64, kSumSlices = 16;

__global__ __launch_bounds__(kSumFeatures * kSumSlices) void sum_partials_kernel(
    const float *__restrict__ dw_parts, const float *__restrict__ db_parts, int64_t H, int blocks,
    float *__restrict__ dw, float *__restrict__ db) {
    __shared__ float s[2][kSumSlices][kSumFeatures];
    const int f = threadIdx.x % kSumFeatures, slice = threadIdx.x / kSumFeatures;
    const int64_t h = int64_t(blockIdx.x) * kSumFeatures + f;
    float w = 0.0f, b = 0.0f;
    if (h < H)
        for (int k = slice; k < blocks; k += kSumSlices) {
            if (dw) w += dw_parts[k * H + h];
            if (db) b += db_parts[k * H + h];
        }
    s[0][slice][f] = w;
    s[1][slice][f] = b;
    __syncthreads();
    if (slice != 0 || h >= H) return;
    for (int k = 1; k < kSumSlices; ++k) {
        w += s[0][k][f];
        b += s[1][k][f];
    }
    if (dw) dw[h] = w;
    if (db) db[h] = b;
}

constexpr int kMaxBlocks = 256;         // rows of partial sums

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

int64_t layer_norm_workspace_bytes(int64_t H, int64_t B) {
    const int64_t blocks = B < kMaxBlocks ? B : kMaxBlocks;
    return 2 * padded(blocks * H * 4);
}

hipError_t launch_layer_norm(int xdtype, int wdtype, int64_t H, int64_t B, const void *x,
                             int64_t x_feature, int64_t x_token, const void *weight,
                             const void *bias, float eps, void *y, int64_t y_feature,
                             int64_t y_token, float *mean, float *rstd, hipStream_t s) {
    const Args a{{const_cast<void *>(x), x_feature, x_token}, {y, y_feature, y_token}, {}, weight,
                 bias, wdtype == DARB_F32, H, B, eps, mean, rstd, nullptr, nullptr};
    return with_type(xdtype, [&](auto type) {
        using T = decltype(type);
        const int64_t blocks = B < 65536 ? B : 65536;
        hipLaunchKernelGGL((any_norm_kernel<T>), dim3(unsigned(blocks)), dim3(kAnyThreads), 0, s, a);
        return hipGetLastError();
    });
}

hipError_t launch_layer_norm_grad(int xdtype, int wdtype, int64_t H, int64_t B, const void *dy,
                                  int64_t dy_feature, int64_t dy_token, const void *x,
                                  int64_t x_feature, int64_t x_token, const float *mean,
                                  const float *rstd, const void *weight, void *dx,
                                  int64_t dx_feature, int64_t dx_token, float *dweight,
                                  float *dbias, void *workspace, hipStream_t s) {
    Args a{{const_cast<void *>(x), x_feature, x_token}, {dx, dx_feature, dx_token},
           {const_cast<void *>(dy), dy_feature, dy_token}, weight, nullptr, wdtype == DARB_F32,
           H, B, 0.0f, const_cast<float *>(mean), const_cast<float *>(rstd), nullptr, nullptr};
    return with_type(xdtype, [&](auto type) {
        using T = decltype(type);
        const int blocks = B < kMaxBlocks ? int(B) : kMaxBlocks;
        if (dweight) a.dw = static_cast<float *>(workspace);
        if (dbias) a.db = reinterpret_cast<float *>(static_cast<char *>(workspace) + padded(blocks * H * 4));
        hipLaunchKernelGGL((any_norm_grad_kernel<T>), dim3(unsigned(blocks)), dim3(kAnyThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || (!dweight && !dbias)) return e;
        hipLaunchKernelGGL(sum_partials_kernel,
                           dim3(unsigned((H + kSumFeatures - 1) / kSumFeatures)),
                           dim3(kSumFeatures * kSumSlices), 0, s, a.dw, a.db, H, blocks, dweight, dbias);
        return hipGetLastError();
    });
}

}  // namespace darb
