// Host side of the calls that evaluate and retrain a DARB layer: argument checks and dispatch.
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "darb_internal.h"

struct darb_adamw {
    int bits = 32;
    int device = -1;
    std::vector<darb::AdamTensor> tensors;
    std::vector<int64_t> first_tile;        // [count + 1]
    darb::AdamTensor *d_tensors = nullptr;  // inside the caller's workspace
    darb::AdamTile *d_tiles = nullptr;
};

namespace darb {
namespace {

constexpr int64_t kMax = int64_t(1) << 31;

bool float_dtype(int t) { return t == DARB_F32 || t == DARB_F16 || t == DARB_BF16; }

bool aligned(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int64_t size_of(int dtype) { return dtype == DARB_F32 ? 4 : 2; }

int check_sizes(int64_t F, int64_t B, const char *name) {
    if (F < 1 || F >= kMax || B < 1 || B >= kMax)
        return fail(DARB_E_INVALID, std::string(name) + " and B must be in [1, 2^31)");
    return DARB_OK;
}

// A [F x B] operand of either order: `rows` (feature stride 1) where the whole call can be.
// The stride of an axis of size 1 is set to what the other order would have.
struct Strides {
    int64_t feature, batch;
};

// The other axis' stride reaches over the unit axis; where that has one element it is `least`.
bool as_rows(const Strides &s, int64_t F, int64_t B, int64_t least) {
    return (F == 1 || s.feature == 1) && (B == 1 || s.batch >= (F > 1 ? F : least));
}
bool as_columns(const Strides &s, int64_t F, int64_t B, int64_t least) {
    return (B == 1 || s.batch == 1) && (F == 1 || s.feature >= (B > 1 ? B : least));
}

// All operands in one order, or an error.  Sets the unused strides of that order.  (One token's
// operands may each have their own feature stride: where one is not 1, all go by columns.)  The
// first `reads` operands are only read, and may repeat one element (a stride of 0) where the unit
// axis has one.
int common_order(Strides *s, int count, int reads, int64_t F, int64_t B, const char *where, bool *by_rows) {
    bool rows = true, columns = true;
    for (int i = 0; i < count; ++i) {
        const int64_t least = i < reads ? 0 : 1;
        rows = rows && as_rows(s[i], F, B, least);
        columns = columns && as_columns(s[i], F, B, least);
    }
    *by_rows = rows;
    if (!rows && !columns)
        return fail(DARB_E_INVALID, std::string(where) + ": one stride must be 1, along the same "
                                    "axis in every operand, and the other at least that axis' length");
    for (int i = 0; i < count; ++i) {
        if (rows) {
            s[i].feature = 1;
        } else {
            s[i].batch = 1;
        }
    }
    return DARB_OK;
}

int check_workspace(const void *workspace, int64_t have, int64_t need) {
    if (!workspace || !aligned(workspace, 256))
        return fail(DARB_E_INVALID, "workspace must be 256-byte aligned device memory");
    if (have < need)
        return fail(DARB_E_WORKSPACE, "workspace needs " + std::to_string(need) + " bytes");
    return DARB_OK;
}

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

int64_t tiles_of(int64_t n) { return (n + adam_tile_elements() - 1) / adam_tile_elements(); }

int check_adamw_table(const darb_adamw_tensor *t, int64_t count, int64_t *tiles) {
    if (!t) return fail(DARB_E_INVALID, "tensors is NULL");
    if (count < 1 || count >= kMax) return fail(DARB_E_INVALID, "count must be in [1, 2^31)");
    *tiles = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n >= int64_t(1) << 39)
            return fail(DARB_E_INVALID, "tensor " + std::to_string(i) + ": n must be in [0, 2^39)");
        *tiles += tiles_of(t[i].n);
    }
    if (*tiles >= kMax) return fail(DARB_E_INVALID, "the tensors have too many elements");
    return DARB_OK;
}

int check_adamw_tensor(const darb_adamw_tensor &t, int64_t i, int bits) {
    const std::string name = "tensor " + std::to_string(i) + ": ";
    if (!float_dtype(t.dtype)) return fail(DARB_E_DTYPE, name + "unknown dtype");
    if (!(t.decay >= 0.0) || !std::isfinite(t.decay))
        return fail(DARB_E_INVALID, name + "decay must be finite and >= 0");
    if (t.n == 0) return DARB_OK;
    if (!t.param || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale)))
        return fail(DARB_E_INVALID, name + "NULL buffer");
    if (!aligned(t.param, size_of(t.dtype)) || !aligned(t.master, 4) || !aligned(t.m_scale, 4) ||
        !aligned(t.v_scale, 4) || (bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))))
        return fail(DARB_E_INVALID, name + "a buffer is not aligned to its elements");
    return DARB_OK;
}

int check_device(const darb_adamw &a) {
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(DARB_E_HIP, std::string("hipGetDevice: ") + hipGetErrorString(e));
    if (dev != a.device)
        return fail(DARB_E_INVALID, "the optimizer was created on device " + std::to_string(a.device) +
                                        ", current device is " + std::to_string(dev));
    return DARB_OK;
}

// The launches of a call over all tensors: f(first tensor, tensors, first tile, tiles) for at most
// `most` tensors and 2^22 tiles each (a launch has below 2^32 threads); a larger tensor takes
// several.
template <typename F> int over_tensors(const darb_adamw &a, int64_t most, F &&f) {
    constexpr int64_t kMostTiles = int64_t(1) << 22;
    const int64_t count = int64_t(a.tensors.size()), all = a.first_tile[count];
    int64_t i = 0;
    for (int64_t tile = 0; tile < all;) {
        while (a.first_tile[i + 1] <= tile) ++i;         // the tensor of this tile
        int64_t end = tile + kMostTiles < all ? tile + kMostTiles : all, j = i + 1;
        while (j < count && j - i < most && a.first_tile[j] < end) ++j;
        if (end > a.first_tile[j]) end = a.first_tile[j];
        const int rc = f(i, j - i, tile, end - tile);
        if (rc) return rc;
        tile = end;
    }
    return DARB_OK;
}

// Whether products are as accurate as fp32: unless the caller takes those of fp16 operands for a 16-bit
// result.  Small matrices are accurate all the same: with single products their results are up to
// 6 10^-3 of the norm off (3 10^-3 from 64 on).  16 matrices of 48 x 48 take 127 us so instead of 123,
// of 48 x 2000 241 instead of 192.
bool muon_full(const darb_muon_tensor &t) {
    return !t.fp16_products || t.dtype == DARB_F32 || t.master || (t.rows < t.cols ? t.rows : t.cols) < 64;
}

// The groups of tensors that go through the launches together: consecutive ones of one accuracy,
// up to kMuonTensors and 4 GiB of their buffers (or a single one).  A tensor that is left out
// (`skip`: without a gradient) counts in its group all the same, so that no step's groups take
// more than those of all tensors.  f(group, its bytes).
template <typename F>
int over_groups(const darb_muon_tensor *t, int64_t count, bool skip, double lr, F &&f) {
    constexpr int64_t kMost = int64_t(1) << 32;
    for (int full = 0; full < 2; ++full) {
        MuonCall c{};
        c.full = full != 0;
        int members = 0;
        int64_t sum = 0;
        for (int64_t i = 0; i <= count; ++i) {
            const bool end = i == count;
            if (!end && muon_full(t[i]) != c.full) continue;
            const int64_t n = end ? 0 : muon_bytes(t[i].rows, t[i].cols);
            if (members && (end || members == kMuonTensors || sum + n > kMost)) {
                if (c.count) {
                    const int64_t bytes = muon_group(c);
                    const int rc = f(c, bytes);
                    if (rc) return rc;
                }
                members = c.count = 0;
                sum = 0;
            }
            if (end) break;
            ++members;
            sum += n;
            if (skip && !t[i].grad) continue;
            MuonTensor &to = c.t[c.count++];
            to = {};
            to.param = t[i].param, to.master = t[i].master, to.grad = t[i].grad, to.momentum = t[i].momentum;
            to.ld_in = t[i].ld_grad, to.ld_out = t[i].ld_param;
            to.rows = int32_t(t[i].rows), to.cols = int32_t(t[i].cols);
            to.dtype = t[i].dtype, to.gdtype = t[i].gdtype;
            to.scale = float(lr * t[i].scale), to.keep = float(1.0 - lr * t[i].decay);
        }
    }
    return DARB_OK;
}

}  // namespace
}  // namespace darb

using namespace darb;

extern "C" {

static int check_logits(int zdtype, int64_t V, int64_t B, int64_t top, Strides *s, bool *rows) {
    int rc = check_sizes(V, B, "V");
    if (rc) return rc;
    if (!float_dtype(zdtype)) return fail(DARB_E_DTYPE, "unknown logit dtype");
    if (top < 0 || top > logprobs_max_top() || top > V)
        return fail(DARB_E_INVALID, "top must be in [0, 64] and at most V");
    return common_order(s, 1, 1, V, B, "z", rows);
}

int darb_token_logprobs_workspace(int zdtype, int64_t V, int64_t B, int64_t z_feature_stride,
                                  int64_t z_batch_stride, int64_t top, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    Strides s[1] = {{z_feature_stride, z_batch_stride}};
    bool rows;
    int rc = check_logits(zdtype, V, B, top, s, &rows);
    if (rc) return rc;
    *bytes = logprobs_workspace_bytes(zdtype, V, B, rows, top);
    return DARB_OK;
}

int darb_token_logprobs(int zdtype, int64_t V, int64_t B, const void *z, int64_t z_feature_stride,
                        int64_t z_batch_stride, const int64_t *targets, int64_t top,
                        float *logprob, float *entropy, float *lse, float *top_logprob,
                        int64_t *top_index, void *workspace, int64_t workspace_bytes,
                        void *stream) {
    clear_error();
    Strides s[1] = {{z_feature_stride, z_batch_stride}};
    bool rows;
    int rc = check_logits(zdtype, V, B, top, s, &rows);
    if (rc) return rc;
    if (!z || !logprob || !entropy || !lse || (top && (!top_logprob || !top_index)))
        return fail(DARB_E_INVALID, "NULL buffer");
    if (!aligned(z, size_of(zdtype)) || !aligned(targets, 8) || !aligned(top_index, 8))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    const int64_t need = logprobs_workspace_bytes(zdtype, V, B, rows, top);
    if (need > 0 && (rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    return launched(launch_logprobs(zdtype, V, B, rows, z, s[0].feature, s[0].batch, targets, top,
                                    logprob, entropy, lse, top_logprob, top_index, workspace,
                                    static_cast<hipStream_t>(stream)), "token logprobs launch");
}

int darb_token_logprobs_grad(int zdtype, int64_t V, int64_t B, const void *z,
                             int64_t z_feature_stride, int64_t z_batch_stride,
                             const int64_t *targets, const float *lse, const float *grad_logprob,
                             const float *entropy, const float *grad_entropy, void *dz,
                             int64_t dz_feature_stride, int64_t dz_batch_stride, void *stream) {
    clear_error();
    int rc = check_sizes(V, B, "V");
    if (rc) return rc;
    if (!float_dtype(zdtype)) return fail(DARB_E_DTYPE, "unknown logit dtype");
    if (!z || !lse || !dz) return fail(DARB_E_INVALID, "NULL buffer");
    if ((entropy == nullptr) != (grad_entropy == nullptr))
        return fail(DARB_E_INVALID, "pass entropy and grad_entropy, or neither");
    if (!grad_logprob && !grad_entropy)
        return fail(DARB_E_INVALID, "pass grad_logprob or grad_entropy");
    if (!aligned(z, size_of(zdtype)) || !aligned(dz, size_of(zdtype)) || !aligned(targets, 8))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    Strides s[2] = {{z_feature_stride, z_batch_stride}, {dz_feature_stride, dz_batch_stride}};
    bool rows;
    rc = common_order(s, 2, 1, V, B, "z, dz", &rows);
    if (rc) return rc;
    return launched(launch_logprobs_grad(zdtype, V, B, rows, z, s[0].feature, s[0].batch, targets, lse,
                                         grad_logprob, entropy, grad_entropy, dz, s[1].feature,
                                         s[1].batch, static_cast<hipStream_t>(stream)),
                    "token logprobs gradient launch");
}

static int check_norm(int xdtype, int wdtype, int64_t H, int64_t B, const void *x,
                      const void *weight, const void *bias) {
    int rc = check_sizes(H, B, "H");
    if (rc) return rc;
    if (!float_dtype(xdtype)) return fail(DARB_E_DTYPE, "unknown activation dtype");
    if (wdtype != DARB_F32 && wdtype != xdtype)
        return fail(DARB_E_DTYPE, "weight and bias must be fp32 or of x's type");
    if (!x) return fail(DARB_E_INVALID, "NULL buffer");
    if (!aligned(x, size_of(xdtype)) || !aligned(weight, size_of(wdtype)) ||
        !aligned(bias, size_of(wdtype)))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    return DARB_OK;
}

int darb_layer_norm(int xdtype, int wdtype, int64_t H, int64_t B, const void *x,
                    int64_t x_feature_stride, int64_t x_batch_stride, const void *weight,
                    const void *bias, double eps, void *y, int64_t y_feature_stride,
                    int64_t y_batch_stride, float *mean, float *rstd, void *stream) {
    clear_error();
    int rc = check_norm(xdtype, wdtype, H, B, x, weight, bias);
    if (rc) return rc;
    if (!y) return fail(DARB_E_INVALID, "NULL buffer");
    if (!aligned(y, size_of(xdtype)))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(DARB_E_INVALID, "eps must be finite and >= 0");
    Strides s[2] = {{x_feature_stride, x_batch_stride}, {y_feature_stride, y_batch_stride}};
    bool rows;
    rc = common_order(s, 2, 1, H, B, "x, y", &rows);
    if (rc) return rc;
    return launched(launch_layer_norm(xdtype, wdtype, H, B, rows, x, s[0].feature, s[0].batch, weight,
                                      bias, float(eps), y, s[1].feature, s[1].batch, mean, rstd,
                                      static_cast<hipStream_t>(stream)), "layer norm launch");
}

int darb_layer_norm_workspace(int64_t H, int64_t B, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    int rc = check_sizes(H, B, "H");
    if (rc) return rc;
    *bytes = layer_norm_workspace_bytes(H, B);
    return DARB_OK;
}

int darb_layer_norm_grad(int xdtype, int wdtype, int64_t H, int64_t B, const void *dy,
                         int64_t dy_feature_stride, int64_t dy_batch_stride, const void *x,
                         int64_t x_feature_stride, int64_t x_batch_stride, const float *mean,
                         const float *rstd, const void *weight, void *dx,
                         int64_t dx_feature_stride, int64_t dx_batch_stride, float *dweight,
                         float *dbias, void *workspace, int64_t workspace_bytes, void *stream) {
    clear_error();
    int rc = check_norm(xdtype, wdtype, H, B, x, weight, nullptr);
    if (rc) return rc;
    if (!dy || !mean || !rstd) return fail(DARB_E_INVALID, "NULL buffer");
    if (!dx && !dweight && !dbias)
        return fail(DARB_E_INVALID, "pass at least one of dx, dweight, dbias");
    if (!aligned(dy, size_of(xdtype)) || !aligned(dx, size_of(xdtype)))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    Strides s[3] = {{x_feature_stride, x_batch_stride}, {dy_feature_stride, dy_batch_stride},
                    {dx_feature_stride, dx_batch_stride}};
    bool rows;
    rc = common_order(s, dx ? 3 : 2, 2, H, B, "x, dy, dx", &rows);
    if (rc) return rc;
    rc = check_workspace(workspace, workspace_bytes, layer_norm_workspace_bytes(H, B));
    if (rc) return rc;
    return launched(launch_layer_norm_grad(xdtype, wdtype, H, B, rows, dy, s[1].feature, s[1].batch, x,
                                           s[0].feature, s[0].batch, mean, rstd, weight, dx,
                                           s[2].feature, s[2].batch, dweight, dbias, workspace,
                                           static_cast<hipStream_t>(stream)),
                    "layer norm gradient launch");
}

static int check_index(const darb_plan *p) {
    if (p->nnz >= kMax) return fail(DARB_E_INVALID, "the plan keeps 2^31 weights or more");
    return DARB_OK;
}

int darb_transpose_bytes(const darb_plan *p, int64_t *bytes) {
    clear_error();
    if (!p || !bytes) return fail(DARB_E_INVALID, "NULL pointer");
    int rc = check_index(p);
    if (rc) return rc;
    *bytes = transpose_bytes(*p);
    return DARB_OK;
}

int darb_transpose(const darb_plan *p, const uint8_t *offsets, void *index, int64_t index_bytes,
                   void *stream) {
    clear_error();
    int rc = check_uploaded(p);
    if (rc) return rc;
    if (!offsets) return fail(DARB_E_INVALID, "NULL buffer");
    rc = check_index(p);
    if (rc) return rc;
    rc = check_workspace(index, index_bytes, transpose_bytes(*p));
    if (rc) return rc;
    return launched(launch_transpose(*p, offsets, index, static_cast<hipStream_t>(stream)),
                    "transpose launch");
}

int darb_spmm_grad_workspace(const darb_plan *p, int64_t B, int64_t *bytes) {
    clear_error();
    if (!p || !bytes) return fail(DARB_E_INVALID, "NULL pointer");
    if (B < 1 || B >= kMax) return fail(DARB_E_INVALID, "B must be in [1, 2^31)");
    int rc = check_index(p);
    if (rc) return rc;
    *bytes = spmm_grad_workspace_bytes(*p, B);
    return DARB_OK;
}

int darb_spmm_grad(const darb_plan *p, const void *index, int wdtype, const void *values,
                   int xdtype, int64_t B, const void *X, int64_t ldx, const float *dY,
                   int64_t ldy, float *dvalues, float *dX, int64_t lddx, void *workspace,
                   int64_t workspace_bytes, void *stream) {
    clear_error();
    int rc = check_uploaded(p);
    if (rc) return rc;
    if ((wdtype != DARB_F32 && wdtype != DARB_F16) || (xdtype != DARB_F32 && xdtype != DARB_F16))
        return fail(DARB_E_DTYPE, "unknown dtype");
    if (wdtype == DARB_F32 && xdtype != DARB_F32)
        return fail(DARB_E_DTYPE, "fp32 weights need fp32 activations");
    if (!index || !dY || (dX && !values) || (dvalues && !X))
        return fail(DARB_E_INVALID, "NULL buffer");
    if (!dvalues && !dX) return fail(DARB_E_INVALID, "pass dvalues or dX");
    if (!aligned(index, 256)) return fail(DARB_E_INVALID, "index must be 256-byte aligned");
    rc = check_index(p);
    if (rc) return rc;
    if (B < 1 || B >= kMax) return fail(DARB_E_INVALID, "B must be in [1, 2^31)");
    if (ldy < B || (dvalues && ldx < B) || (dX && lddx < B))
        return fail(DARB_E_INVALID, "a leading dimension is below B");
    const int64_t need = spmm_grad_workspace_bytes(*p, B);
    if (need > 0 && (rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    return launched(launch_spmm_grad(*p, index, wdtype, values, xdtype, B, X, ldx, dY, ldy,
                                     dvalues, dX, lddx, workspace, static_cast<hipStream_t>(stream)),
                    "spmm gradient launch");
}

int darb_adamw_workspace(const darb_adamw_tensor *tensors, int64_t count, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    int64_t tiles;
    int rc = check_adamw_table(tensors, count, &tiles);
    if (rc) return rc;
    *bytes = padded(count * int64_t(sizeof(AdamTensor))) + padded(tiles * int64_t(sizeof(AdamTile)));
    return DARB_OK;
}

int darb_adamw_create(const darb_adamw_tensor *tensors, int64_t count, int bits, void *workspace,
                      int64_t workspace_bytes, void *stream, darb_adamw **out) {
    clear_error();
    if (!out) return fail(DARB_E_INVALID, "out is NULL");
    *out = nullptr;
    if (bits != 32 && bits != 8) return fail(DARB_E_INVALID, "bits must be 32 or 8");
    int64_t tiles;
    int rc = check_adamw_table(tensors, count, &tiles);
    if (rc) return rc;
    for (int64_t i = 0; i < count; ++i)
        if ((rc = check_adamw_tensor(tensors[i], i, bits))) return rc;
    const int64_t table = padded(count * int64_t(sizeof(AdamTensor)));
    rc = check_workspace(workspace, workspace_bytes, table + padded(tiles * int64_t(sizeof(AdamTile))));
    if (rc) return rc;
    darb_adamw *a = new (std::nothrow) darb_adamw();
    if (!a) return fail(DARB_E_NOMEM, "optimizer handle");
    std::vector<AdamTile> list;
    try {
        a->bits = bits;
        a->tensors.resize(count);
        a->first_tile.resize(count + 1);
        list.resize(tiles);
    } catch (const std::bad_alloc &) {
        delete a;
        return fail(DARB_E_NOMEM, "optimizer tables");
    }
    int64_t at = 0;
    for (int64_t i = 0; i < count; ++i) {
        const darb_adamw_tensor &t = tensors[i];
        a->tensors[i] = {t.param, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n, t.decay, t.dtype, 0};
        a->first_tile[i] = at;
        for (int64_t k = 0; k < tiles_of(t.n); ++k) list[at++] = {uint32_t(i), uint32_t(k)};
    }
    a->first_tile[count] = at;
    if (hipGetDevice(&a->device) != hipSuccess) {
        delete a;
        (void)hipGetLastError();
        return fail(DARB_E_HIP, "hipGetDevice failed");
    }
    a->d_tensors = static_cast<AdamTensor *>(workspace);
    a->d_tiles = reinterpret_cast<AdamTile *>(static_cast<char *>(workspace) + table);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipMemcpyAsync(a->d_tensors, a->tensors.data(), count * sizeof(AdamTensor),
                                  hipMemcpyHostToDevice, s);
    if (e == hipSuccess && tiles)
        e = hipMemcpyAsync(a->d_tiles, list.data(), tiles * sizeof(AdamTile), hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) {
        delete a;
        (void)hipGetLastError();
        return fail(DARB_E_HIP, std::string("optimizer tables: ") + hipGetErrorString(e));
    }
    *out = a;
    return DARB_OK;
}

int darb_adamw_step(const darb_adamw *a, const void *const *grads, const int *gdtypes,
                    int64_t count, double lr, double beta1, double beta2, double eps,
                    int64_t step, const float *grad_scale, uint32_t seed, void *stream) {
    clear_error();
    if (!a || !grads || !gdtypes) return fail(DARB_E_INVALID, "NULL pointer");
    if (count != int64_t(a->tensors.size()))
        return fail(DARB_E_INVALID, "the optimizer has " + std::to_string(a->tensors.size()) + " tensors");
    if (!(lr >= 0.0) || !std::isfinite(lr) || !(eps >= 0.0) || !std::isfinite(eps))
        return fail(DARB_E_INVALID, "lr and eps must be finite and >= 0");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
        return fail(DARB_E_INVALID, "beta1 and beta2 must be in [0, 1)");
    if (step < 1) return fail(DARB_E_INVALID, "step must be >= 1");
    if (!aligned(grad_scale, 4)) return fail(DARB_E_INVALID, "grad_scale is not aligned");
    for (int64_t i = 0; i < count; ++i) {
        if (!grads[i]) continue;
        if (!float_dtype(gdtypes[i]))
            return fail(DARB_E_DTYPE, "gradient " + std::to_string(i) + ": unknown dtype");
        if (!aligned(grads[i], size_of(gdtypes[i])))
            return fail(DARB_E_INVALID, "gradient " + std::to_string(i) + " is not aligned to its elements");
    }
    const int rc = check_device(*a);
    if (rc) return rc;
    const AdamScalars k{lr, beta1, beta2, eps, step, grad_scale, seed};
    return over_tensors(*a, kAdamGrads, [&](int64_t i, int64_t n, int64_t tile, int64_t tiles) {
        return launched(launch_adamw(a->bits, a->d_tensors, a->d_tiles + tile, tiles, int(i), int(n),
                                     grads + i, gdtypes + i, k, static_cast<hipStream_t>(stream)),
                        "adamw launch");
    });
}

int darb_adamw_moments(const darb_adamw *a, float *const *m, float *const *v, int64_t count,
                       void *stream) {
    clear_error();
    if (!a) return fail(DARB_E_INVALID, "NULL pointer");
    if (count != int64_t(a->tensors.size()))
        return fail(DARB_E_INVALID, "the optimizer has " + std::to_string(a->tensors.size()) + " tensors");
    for (int64_t i = 0; i < count; ++i)
        if (!aligned(m ? m[i] : nullptr, 4) || !aligned(v ? v[i] : nullptr, 4))
            return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    const int rc = check_device(*a);
    if (rc) return rc;
    return over_tensors(*a, kAdamGrads / 2, [&](int64_t i, int64_t n, int64_t tile, int64_t tiles) {
        return launched(launch_moments(a->bits, a->d_tensors, a->d_tiles + tile, tiles, int(i),
                                       int(n), m ? m + i : nullptr, v ? v + i : nullptr,
                                       static_cast<hipStream_t>(stream)), "moments launch");
    });
}

void darb_adamw_destroy(darb_adamw *a) { delete a; }

static bool recurrence_sizes(int64_t H, int64_t T, int64_t batch) {
    return H >= 1 && H < kMax && T >= 1 && batch >= 1 && T < kMax && batch < kMax && T * batch < kMax;
}

static int check_recurrence(int dtype, int form, int64_t H, int64_t T, int64_t batch) {
    if (!recurrence_sizes(H, T, batch))
        return fail(DARB_E_INVALID, "H, T and batch must be >= 1, H and T * batch below 2^31");
    if (!float_dtype(dtype)) return fail(DARB_E_DTYPE, "unknown dtype");
    if (form != DARB_RECURRENCE_GATE && form != DARB_RECURRENCE_LINEAR)
        return fail(DARB_E_INVALID, "unknown form");
    return DARB_OK;
}

static int64_t recurrence_bytes(int dtype, bool back, int64_t H, int64_t T, int64_t batch) {
    const int64_t a = recurrence_workspace_bytes(dtype, back, false, H, T, batch);
    const int64_t b = recurrence_workspace_bytes(dtype, back, true, H, T, batch);
    return a > b ? a : b;
}

// A state [H x batch] of either order; `read`: its elements may coincide.
static int check_state(const darb_matrix *m, bool read, int64_t H, int64_t batch, const char *name,
                       RecurrenceMatrix *out) {
    if (!m || !m->p) return DARB_OK;
    if (!aligned(m->p, 4)) return fail(DARB_E_INVALID, std::string(name) + " is not aligned to its elements");
    const Strides s{m->feature_stride, m->batch_stride};
    if (s.feature < 0 || s.batch < 0 ||
        (!read && !as_rows(s, H, batch, 1) && !as_columns(s, H, batch, 1)))
        return fail(DARB_E_INVALID, std::string(name) + ": one stride must be 1 and the other at least that axis' length");
    *out = {m->p, s.feature, s.batch};
    return DARB_OK;
}

// The operands [H x T*batch], all in one order; `reads` of them are only read.
static int check_sequences(RecurrenceMatrix *const *to, const darb_matrix *const *m, int count, int reads, int64_t H,
                           int64_t columns, int dtype, const char *where, bool *rows) {
    Strides s[6];
    for (int i = 0; i < count; ++i) {
        if (!m[i] || !m[i]->p) return fail(DARB_E_INVALID, "NULL buffer");
        if (!aligned(m[i]->p, size_of(dtype))) return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
        s[i] = {m[i]->feature_stride, m[i]->batch_stride};
    }
    const int rc = common_order(s, count, reads, H, columns, where, rows);
    if (rc) return rc;
    for (int i = 0; i < count; ++i) *to[i] = {m[i]->p, s[i].feature, s[i].batch};
    return DARB_OK;
}

int darb_gated_recurrence_workspace(int dtype, int back, int64_t H, int64_t T, int64_t batch, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    const int rc = check_recurrence(dtype, DARB_RECURRENCE_GATE, H, T, batch);
    if (rc) return rc;
    *bytes = recurrence_bytes(dtype, back != 0, H, T, batch);
    return DARB_OK;
}

int darb_gated_recurrence(int dtype, int form, int64_t H, int64_t T, int64_t batch, const darb_matrix *gate,
                          const darb_matrix *x, const uint8_t *resets, const darb_matrix *h0, const darb_matrix *h,
                          const darb_matrix *h_last, void *workspace, int64_t workspace_bytes, void *stream) {
    clear_error();
    int rc = check_recurrence(dtype, form, H, T, batch);
    if (rc) return rc;
    RecurrenceCall c;
    const darb_matrix *const m[] = {gate, x, h};
    RecurrenceMatrix *const to[] = {&c.gate, &c.x, &c.out};
    if ((rc = check_sequences(to, m, 3, 2, H, T * batch, dtype, "gate, x, h", &c.rows)) ||
        (rc = check_state(h0, true, H, batch, "h0", &c.in)) ||
        (rc = check_state(h_last, false, H, batch, "h_last", &c.last)))
        return rc;
    const int64_t need = recurrence_bytes(dtype, false, H, T, batch);
    if (need > 0 && (rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    c.dtype = dtype, c.form = form, c.back = false;
    c.H = H, c.T = T, c.batch = batch;
    c.resets = resets, c.workspace = workspace;
    return launched(launch_recurrence(c, static_cast<hipStream_t>(stream)), "gated recurrence launch");
}

int darb_gated_recurrence_grad(int dtype, int form, int64_t H, int64_t T, int64_t batch, const darb_matrix *dh,
                               const darb_matrix *gate, const darb_matrix *x, const darb_matrix *h,
                               const uint8_t *resets, const darb_matrix *h0, const darb_matrix *dh_last,
                               const darb_matrix *dgate, const darb_matrix *dx, const darb_matrix *dh0,
                               void *workspace, int64_t workspace_bytes, void *stream) {
    clear_error();
    int rc = check_recurrence(dtype, form, H, T, batch);
    if (rc) return rc;
    RecurrenceCall c;
    const bool with_x = form == DARB_RECURRENCE_GATE;
    const darb_matrix *const m[] = {dh, gate, h, with_x ? x : gate, dgate, dx};
    RecurrenceMatrix *const to[] = {&c.dh, &c.gate, &c.h, &c.x, &c.out, &c.out2};
    if ((rc = check_sequences(to, m, 6, 4, H, T * batch, dtype, "dh, gate, x, h, dgate, dx", &c.rows)) ||
        (rc = check_state(h0, true, H, batch, "h0", &c.h0)) ||
        (rc = check_state(dh_last, true, H, batch, "dh_last", &c.in)) ||
        (rc = check_state(dh0, false, H, batch, "dh0", &c.last)))
        return rc;
    if (dgate->p == h->p || dx->p == h->p || dgate->p == dx->p)
        return fail(DARB_E_INVALID, "dgate, dx and h must be different buffers");
    const int64_t need = recurrence_bytes(dtype, true, H, T, batch);
    if (need > 0 && (rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    c.dtype = dtype, c.form = form, c.back = true;
    c.H = H, c.T = T, c.batch = batch;
    c.resets = resets, c.workspace = workspace;
    return launched(launch_recurrence(c, static_cast<hipStream_t>(stream)), "gated recurrence gradient launch");
}

int darb_policy_loss_workspace(int64_t B, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    if (B < 1 || B >= kMax) return fail(DARB_E_INVALID, "B must be in [1, 2^31)");
    *bytes = policy_workspace_bytes(B);
    return DARB_OK;
}

int darb_policy_loss(int64_t B, const float *logprob, const float *old, const float *advantage, const float *weight,
                     const float *ref, const float *entropy, double clip_low, double clip_high, double kl_coef,
                     double entropy_coef, float *stats, float *grad_logprob, float *grad_entropy, void *workspace,
                     int64_t workspace_bytes, void *stream) {
    clear_error();
    if (B < 1 || B >= kMax) return fail(DARB_E_INVALID, "B must be in [1, 2^31)");
    if (!logprob || !old || !advantage || !stats || !grad_logprob) return fail(DARB_E_INVALID, "NULL buffer");
    if ((entropy == nullptr) != (grad_entropy == nullptr))
        return fail(DARB_E_INVALID, "pass entropy and grad_entropy, or neither");
    if (!(clip_low >= 0.0) || !(clip_high >= 0.0) || !std::isfinite(clip_low) || !std::isfinite(clip_high))
        return fail(DARB_E_INVALID, "clip_low and clip_high must be finite and >= 0");
    if (!(kl_coef >= 0.0) || !std::isfinite(kl_coef) || !std::isfinite(entropy_coef))
        return fail(DARB_E_INVALID, "kl_coef must be finite and >= 0, entropy_coef finite");
    if ((!ref && kl_coef != 0.0) || (!entropy && entropy_coef != 0.0))
        return fail(DARB_E_INVALID, "a coefficient without its values");
    for (const void *p : {static_cast<const void *>(logprob), static_cast<const void *>(old),
                          static_cast<const void *>(advantage), static_cast<const void *>(weight),
                          static_cast<const void *>(ref), static_cast<const void *>(entropy),
                          static_cast<const void *>(stats), static_cast<const void *>(grad_logprob),
                          static_cast<const void *>(grad_entropy)})
        if (!aligned(p, 4)) return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    if (grad_logprob == grad_entropy) return fail(DARB_E_INVALID, "the gradients must be different buffers");
    const int64_t need = policy_workspace_bytes(B);
    int rc;
    if (need > 0 && (rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    PolicyCall c{};
    c.B = B;
    c.lp = logprob, c.old = old, c.advantage = advantage, c.weight = weight, c.ref = ref, c.entropy = entropy;
    c.grad = grad_logprob, c.grad_entropy = grad_entropy, c.stats = stats;
    c.partial = static_cast<double *>(workspace);
    c.even = float(1.0 / double(B));
    c.low = float(1.0 - clip_low), c.high = float(1.0 + clip_high);
    c.kl_coef = float(kl_coef), c.entropy_coef = float(entropy_coef);
    c.log_low = clip_low < 1.0 ? std::log1p(-clip_low) : -HUGE_VAL;
    c.log_high = std::log1p(clip_high);
    return launched(launch_policy(c, static_cast<hipStream_t>(stream)), "policy loss launch");
}

int darb_preference_loss(int64_t pairs, int64_t B, const float *logprob, const float *ref, const int64_t *starts,
                         const float *weight, double beta, double smoothing, float *loss, float *margin,
                         float *grad_logprob, void *stream) {
    clear_error();
    if (pairs < 1 || pairs >= kMax / 2) return fail(DARB_E_INVALID, "pairs must be in [1, 2^30)");
    if (B < 1 || B >= kMax) return fail(DARB_E_INVALID, "B must be in [1, 2^31)");
    if (!starts && B % (2 * pairs) != 0) return fail(DARB_E_INVALID, "B must be a multiple of 2 * pairs");
    if (!logprob || !loss || !margin || !grad_logprob) return fail(DARB_E_INVALID, "NULL buffer");
    if (!(beta >= 0.0) || !std::isfinite(beta)) return fail(DARB_E_INVALID, "beta must be finite and >= 0");
    if (!(smoothing >= 0.0 && smoothing < 1.0)) return fail(DARB_E_INVALID, "smoothing must be in [0, 1)");
    if (!aligned(logprob, 4) || !aligned(ref, 4) || !aligned(starts, 8) || !aligned(weight, 4) || !aligned(loss, 4) ||
        !aligned(margin, 4) || !aligned(grad_logprob, 4))
        return fail(DARB_E_INVALID, "a buffer is not aligned to its elements");
    PreferenceCall c{};
    c.P = pairs, c.B = B, c.L = B / (2 * pairs);
    c.lp = logprob, c.ref = ref, c.weight = weight, c.starts = starts;
    c.loss = loss, c.margin = margin, c.grad = grad_logprob;
    c.even = float(1.0 / double(pairs)), c.beta = float(beta), c.smoothing = float(smoothing);
    return launched(launch_preference(c, static_cast<hipStream_t>(stream)), "preference loss launch");
}

static int check_muon(const darb_muon_tensor *t, int64_t count, bool buffers, bool update) {
    if (!t) return fail(DARB_E_INVALID, "tensors is NULL");
    if (count < 1 || count >= kMax) return fail(DARB_E_INVALID, "count must be in [1, 2^31)");
    for (int64_t i = 0; i < count; ++i) {
        const std::string name = "tensor " + std::to_string(i) + ": ";
        if (t[i].rows < 1 || t[i].rows >= int64_t(1) << 20 || t[i].cols < 1 || t[i].cols >= int64_t(1) << 20)
            return fail(DARB_E_INVALID, name + "rows and cols must be in [1, 2^20)");
        if (!float_dtype(t[i].dtype)) return fail(DARB_E_DTYPE, name + "unknown dtype");
        if (t[i].fp16_products < 0 || t[i].fp16_products > 1 || t[i].reserved != 0)
            return fail(DARB_E_INVALID, name + "fp16_products must be 0 or 1, reserved 0");
        if (!buffers) continue;
        if (t[i].ld_param < t[i].cols) return fail(DARB_E_INVALID, name + "a leading dimension is below cols");
        if (!t[i].param || (update && !t[i].momentum)) return fail(DARB_E_INVALID, name + "NULL buffer");
        if (!update && !t[i].grad) return fail(DARB_E_INVALID, name + "NULL buffer");
        if (!aligned(t[i].param, size_of(t[i].dtype)) || !aligned(t[i].master, 4) || !aligned(t[i].momentum, 4))
            return fail(DARB_E_INVALID, name + "a buffer is not aligned to its elements");
        if (update && (!std::isfinite(t[i].scale) || !(t[i].decay >= 0.0) || !std::isfinite(t[i].decay)))
            return fail(DARB_E_INVALID, name + "scale must be finite, decay finite and >= 0");
        if (!t[i].grad) continue;
        if (!float_dtype(t[i].gdtype)) return fail(DARB_E_DTYPE, name + "unknown gradient dtype");
        if (t[i].ld_grad < t[i].cols) return fail(DARB_E_INVALID, name + "a leading dimension is below cols");
        if (!aligned(t[i].grad, size_of(t[i].gdtype)))
            return fail(DARB_E_INVALID, name + "a buffer is not aligned to its elements");
    }
    return DARB_OK;
}

int darb_muon_workspace(const darb_muon_tensor *tensors, int64_t count, int64_t *bytes) {
    clear_error();
    if (!bytes) return fail(DARB_E_INVALID, "bytes is NULL");
    int rc = check_muon(tensors, count, false, false);
    if (rc) return rc;
    *bytes = 0;
    return over_groups(tensors, count, false, 0.0, [&](MuonCall &, int64_t need) {
        if (need > *bytes) *bytes = need;
        return int(DARB_OK);
    });
}

static int muon(const darb_muon_tensor *tensors, int64_t count, bool update, double lr, double momentum, int nesterov,
                int steps, double eps, const float *grad_scale, void *workspace, int64_t workspace_bytes,
                void *stream, const int *kinds = nullptr) {
    if (steps < 1 || steps > 16) return fail(DARB_E_INVALID, "steps must be in [1, 16]");
    if (!(eps > 0.0) || !std::isfinite(eps)) return fail(DARB_E_INVALID, "eps must be finite and > 0");
    if (!(lr >= 0.0) || !std::isfinite(lr)) return fail(DARB_E_INVALID, "lr must be finite and >= 0");
    if (!(momentum >= 0.0 && momentum < 1.0)) return fail(DARB_E_INVALID, "momentum must be in [0, 1)");
    if (!aligned(grad_scale, 4)) return fail(DARB_E_INVALID, "grad_scale is not aligned");
    int rc = check_muon(tensors, count, true, update);
    if (rc) return rc;
    rc = check_workspace(workspace, workspace_bytes, 0);
    if (rc) return rc;
    auto group = [&](MuonCall &c, int64_t bytes) {
        if (bytes > workspace_bytes)
            return fail(DARB_E_WORKSPACE, "workspace needs " + std::to_string(bytes) + " bytes");
        return int(DARB_OK);
    };
    if ((rc = over_groups(tensors, count, update, lr, group))) return rc;       // all, before the first launch
    return over_groups(tensors, count, update, lr, [&](MuonCall &c, int64_t) {
        c.update = update;
        c.nesterov = nesterov != 0;
        c.steps = steps;
        c.mu = float(momentum), c.one_mu = float(1.0 - momentum);
        c.eps = eps;
        c.grad_scale = grad_scale;
        c.workspace = workspace;
        for (int i = 0; kinds && i < 3; ++i) c.kind[i] = int8_t(kinds[i]);
        return launched(launch_muon(c, static_cast<hipStream_t>(stream)), "orthogonalised update launch");
    });
}

int darb_muon_step(const darb_muon_tensor *tensors, int64_t count, double lr, double momentum, int nesterov,
                   int steps, double eps, const float *grad_scale, void *workspace, int64_t workspace_bytes,
                   void *stream) {
    clear_error();
    return muon(tensors, count, true, lr, momentum, nesterov, steps, eps, grad_scale, workspace, workspace_bytes,
                stream);
}

int darb_orthogonalize(const darb_muon_tensor *tensors, int64_t count, int steps, double eps, void *workspace,
                       int64_t workspace_bytes, void *stream) {
    clear_error();
    return muon(tensors, count, false, 0.0, 0.0, 0, steps, eps, nullptr, workspace, workspace_bytes, stream);
}

int darb_test_orthogonalize(const darb_muon_tensor *tensors, int64_t count, int steps, double eps, void *workspace,
                            int64_t workspace_bytes, int gram, int square, int apply, void *stream) {
    clear_error();
    const int kinds[3] = {gram, square, apply};
    for (int k : kinds)
        if (k < 0 || k > 4) return fail(DARB_E_INVALID, "unknown tiles");
    if (gram == 1 || square == 1) return fail(DARB_E_INVALID, "tiles on the diagonal are square");
    return muon(tensors, count, false, 0.0, 0.0, 0, steps, eps, nullptr, workspace, workspace_bytes, stream, kinds);
}

}  // extern "C"
