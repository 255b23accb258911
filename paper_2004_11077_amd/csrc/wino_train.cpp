// C ABI of the operators of a training step: argument checks and launches.
#include <cmath>

#include "../../include/wino.h"
#include "wino_kernels.hpp"
#include "wino_train_rules.hpp"

using namespace wino;

namespace {

template <class... A>
int refuse(int code, const char* fmt, A... args) {
  return report_error(code, fmt, args...);
}

int failed(hipError_t e, const char* what) {
  return e == hipSuccess ? WINO_OK : refuse(WINO_EHIP, "%s: %s", what, hipGetErrorString(e));
}

int present(const void* p, const char* name) {
  return p ? WINO_OK : refuse(WINO_EINVAL, "null pointer: %s", name);
}

// Elements start where their own size allows.
int on_element(const void* p, size_t size, const char* name) {
  return (uintptr_t)p % size == 0 ? WINO_OK : refuse(WINO_EINVAL, "%s must be %zu-byte aligned", name, size);
}

int room(const void* ws, size_t have, size_t want) {
  if (int rc = present(ws, "workspace")) return rc;
  if (have < want) return refuse(WINO_EWORKSPACE, "workspace has %zu bytes, %zu needed", have, want);
  if ((uintptr_t)ws % 256) return refuse(WINO_EWORKSPACE, "%s", "workspace must be 256-byte aligned");
  return WINO_OK;
}

size_t size_of(int type) { return type == WINO_TYPE_F32 ? 4 : type == WINO_TYPE_BF16 ? 2 : 1; }
bool real_type(int t) { return t == WINO_TYPE_F32 || t == WINO_TYPE_BF16; }
bool positive(float v) { return std::isfinite(v) && v > 0; }

int stride_of(int64_t given, int64_t row, const char* name, long* out) {
  if (given != 0 && given < row) return refuse(WINO_EINVAL, "%s is smaller than a row", name);
  if (given > (int64_t)1 << 40) return refuse(WINO_EINVAL, "%s is too large", name);
  *out = given ? given : row;
  return WINO_OK;
}

int norm_args(const wino_norm_desc_t* d, NormArgs* a) {
  if (int rc = present(d, "desc")) return rc;
  if (d->rows < 0 || d->rows > (int64_t)1 << 40) return refuse(WINO_EINVAL, "bad rows %lld", (long long)d->rows);
  if (d->channels < 1 || d->channels > 1 << 24) return refuse(WINO_EINVAL, "bad channels %d", d->channels);
  if (!real_type(d->x_type) || !real_type(d->g_type))
    return refuse(WINO_EUNSUPPORTED, "%s", "x_type and g_type are WINO_TYPE_F32 or WINO_TYPE_BF16");
  if (!real_type(d->y_type) && d->y_type != WINO_TYPE_I8)
    return refuse(WINO_EUNSUPPORTED, "unknown y_type %d", d->y_type);
  if (!std::isfinite(d->eps) || d->eps < 0) return refuse(WINO_EINVAL, "%s", "eps must be finite and not negative");
  if (d->y_type == WINO_TYPE_I8 && !positive(d->s_y))
    return refuse(WINO_EINVAL, "%s", "s_y must be positive and finite");
  const double s = d->y_type == WINO_TYPE_I8 ? (double)d->s_y : 1.0;
  *a = NormArgs{(long)d->rows, d->channels, d->x_type, d->y_type, d->g_type, d->eps, s, 1.0 / s,
                1.0 / d->channels, 0, 0, 0, 0};
  if (int rc = stride_of(d->x_stride, d->channels, "x_stride", &a->x_stride)) return rc;
  if (int rc = stride_of(d->y_stride, d->channels, "y_stride", &a->y_stride)) return rc;
  if (int rc = stride_of(d->dy_stride, d->channels, "dy_stride", &a->dy_stride)) return rc;
  return stride_of(d->dx_stride, d->channels, "dx_stride", &a->dx_stride);
}

int loss_args(const wino_loss_desc_t* d, LossArgs* a) {
  if (int rc = present(d, "desc")) return rc;
  if (d->rows < 0 || d->rows > WINO_LOSS_MAX_ROWS) return refuse(WINO_EINVAL, "bad rows %d", d->rows);
  if (d->features < 1 || d->features > WINO_LOSS_MAX_FEATURES)
    return refuse(WINO_EINVAL, "bad features %d", d->features);
  if (d->classes < 1 || d->classes > WINO_LOSS_MAX_CLASSES) return refuse(WINO_EINVAL, "bad classes %d", d->classes);
  if (!real_type(d->type)) return refuse(WINO_EUNSUPPORTED, "%s", "type is WINO_TYPE_F32 or WINO_TYPE_BF16");
  if (d->piece < 0 || d->piece > WINO_LOSS_MAX_ROWS) return refuse(WINO_EINVAL, "bad piece %d", d->piece);
  *a = LossArgs{d->rows, d->features, d->classes, d->type == WINO_TYPE_BF16, 0, 0, (long)d->ignore_index, d->piece};
  if (int rc = stride_of(d->h_stride, d->features, "h_stride", &a->h_stride)) return rc;
  return stride_of(d->w_stride, d->features, "w_stride", &a->w_stride);
}

int update_args(const wino_orthogonalise_desc_t* d, UpdateArgs* a) {
  if (int rc = present(d, "desc")) return rc;
  if (d->batch < 0 || d->batch > 65535) return refuse(WINO_EINVAL, "bad batch %d", d->batch);
  if (d->rows < 0 || d->cols < 0 || d->rows > WINO_ORTHOGONALISE_MAX_SIDE || d->cols > WINO_ORTHOGONALISE_MAX_SIDE)
    return refuse(WINO_EINVAL, "bad matrix %d x %d", d->rows, d->cols);
  // a launch holds fewer than 2^32 threads, 256 a tile of 64 x 64
  if ((int64_t)d->batch * ((d->rows + 63) / 64) * ((d->cols + 63) / 64) > 1 << 23)
    return refuse(WINO_EINVAL, "%d matrices of %d x %d are too many", d->batch, d->rows, d->cols);
  if (!real_type(d->g_type) || !real_type(d->o_type))
    return refuse(WINO_EUNSUPPORTED, "%s", "g_type and o_type are WINO_TYPE_F32 or WINO_TYPE_BF16");
  if (d->steps < 1 || d->steps > 100) return refuse(WINO_EINVAL, "bad steps %d", d->steps);
  if (!std::isfinite(d->a) || !std::isfinite(d->b) || !std::isfinite(d->c) || !std::isfinite(d->scale))
    return refuse(WINO_EINVAL, "%s", "coefficients and scale must be finite");
  if (!positive(d->eps)) return refuse(WINO_EINVAL, "%s", "eps must be positive and finite");
  *a = UpdateArgs{d->batch, d->rows, d->cols, d->g_type == WINO_TYPE_BF16, d->o_type == WINO_TYPE_BF16, d->steps,
                  d->a, d->b, d->c, d->eps, d->scale, 0, 0, 0, 0};
  if (int rc = stride_of(d->g_stride, d->cols, "g_stride", &a->g_stride)) return rc;
  if (int rc = stride_of(d->o_stride, d->cols, "o_stride", &a->o_stride)) return rc;
  const int64_t g_all = d->rows ? (d->rows - 1) * a->g_stride + d->cols : 0;
  const int64_t o_all = d->rows ? (d->rows - 1) * a->o_stride + d->cols : 0;
  if (int rc = stride_of(d->g_batch, g_all, "g_batch", &a->g_batch)) return rc;
  if (!d->g_batch) a->g_batch = d->rows * a->g_stride;
  if (int rc = stride_of(d->o_batch, o_all, "o_batch", &a->o_batch)) return rc;
  if (!d->o_batch) a->o_batch = d->rows * a->o_stride;
  return WINO_OK;
}

}  // namespace

extern "C" {

int wino_layer_norm(const wino_norm_desc_t* d, const void* x, const void* gamma, const void* beta, void* y,
                    void* mean, void* rstd, void* hip_stream) {
  NormArgs a;
  if (int rc = norm_args(d, &a)) return rc;
  if (a.rows == 0) return WINO_OK;
  if (int rc = present(x, "x")) return rc;
  if (int rc = present(y, "y")) return rc;
  if (int rc = on_element(x, size_of(a.x_type), "x")) return rc;
  if (int rc = on_element(y, size_of(a.y_type), "y")) return rc;
  const void* fp32[] = {gamma, beta, mean, rstd};
  const char* names[] = {"gamma", "beta", "mean", "rstd"};
  for (int i = 0; i < 4; ++i)
    if (int rc = on_element(fp32[i], 4, names[i])) return rc;
  return failed(launch_norm(a, x, (const float*)gamma, (const float*)beta, y, (float*)mean, (float*)rstd,
                            (hipStream_t)hip_stream), "layer norm launch");
}

int wino_layer_norm_backward_workspace_bytes(const wino_norm_desc_t* d, size_t* bytes) {
  NormArgs a;
  if (int rc = norm_args(d, &a)) return rc;
  if (!bytes) return refuse(WINO_EINVAL, "%s", "null bytes");
  *bytes = up((size_t)norm_parts(a.rows, a.channels) * 2 * a.channels * 4, 256);
  return WINO_OK;
}

int wino_layer_norm_backward(const wino_norm_desc_t* d, const void* dy, const void* x, const void* gamma,
                             const void* mean, const void* rstd, void* dx, void* dgamma, void* dbeta,
                             void* workspace, size_t ws_bytes, void* hip_stream) {
  NormArgs a;
  if (int rc = norm_args(d, &a)) return rc;
  size_t want = 0;
  if (int rc = wino_layer_norm_backward_workspace_bytes(d, &want)) return rc;
  if (!dx && !dgamma && !dbeta) return WINO_OK;
  if (a.rows != 0) {
    const void* given[] = {dy, x, mean, rstd};
    const char* names[] = {"dy", "x", "mean", "rstd"};
    for (int i = 0; i < 4; ++i)
      if (int rc = present(given[i], names[i])) return rc;
  }
  if (int rc = on_element(dy, size_of(a.g_type), "dy")) return rc;
  if (int rc = on_element(dx, size_of(a.g_type), "dx")) return rc;
  if (int rc = on_element(x, size_of(a.x_type), "x")) return rc;
  const void* fp32[] = {gamma, mean, rstd, dgamma, dbeta};
  const char* names[] = {"gamma", "mean", "rstd", "dgamma", "dbeta"};
  for (int i = 0; i < 5; ++i)
    if (int rc = on_element(fp32[i], 4, names[i])) return rc;
  if (a.rows == 0 && !dgamma && !dbeta) return WINO_OK;
  if (dgamma || dbeta)
    if (int rc = room(workspace, ws_bytes, want)) return rc;
  return failed(launch_norm_backward(a, dy, x, (const float*)gamma, (const float*)mean, (const float*)rstd, dx,
                                     (float*)dgamma, (float*)dbeta, (float*)workspace, (hipStream_t)hip_stream),
                "layer norm backward launch");
}

int wino_linear_cross_entropy_workspace_bytes(const wino_loss_desc_t* d, size_t* bytes) {
  LossArgs a;
  if (int rc = loss_args(d, &a)) return rc;
  if (!bytes) return refuse(WINO_EINVAL, "%s", "null bytes");
  *bytes = loss_layout(a, false).bytes;
  return WINO_OK;
}

int wino_linear_cross_entropy_backward_workspace_bytes(const wino_loss_desc_t* d, size_t* bytes) {
  LossArgs a;
  if (int rc = loss_args(d, &a)) return rc;
  if (!bytes) return refuse(WINO_EINVAL, "%s", "null bytes");
  *bytes = loss_layout(a, true).bytes;
  return WINO_OK;
}

int wino_linear_cross_entropy(const wino_loss_desc_t* d, const void* h, const void* w, const void* bias,
                              const void* targets, void* loss, void* lse, void* workspace, size_t ws_bytes,
                              void* hip_stream) {
  LossArgs a;
  if (int rc = loss_args(d, &a)) return rc;
  if (a.rows == 0) return WINO_OK;
  const void* given[] = {h, w, targets, loss, lse};
  const char* names[] = {"h", "w", "targets", "loss", "lse"};
  const size_t sizes[] = {size_of(d->type), size_of(d->type), 8, 4, 4};
  for (int i = 0; i < 5; ++i) {
    if (int rc = present(given[i], names[i])) return rc;
    if (int rc = on_element(given[i], sizes[i], names[i])) return rc;
  }
  if (int rc = on_element(bias, 4, "bias")) return rc;
  if (int rc = room(workspace, ws_bytes, loss_layout(a, false).bytes)) return rc;
  return failed(launch_loss(a, h, w, (const float*)bias, (const int64_t*)targets, (float*)loss, (float*)lse,
                            (char*)workspace, (hipStream_t)hip_stream), "cross entropy launch");
}

int wino_linear_cross_entropy_backward(const wino_loss_desc_t* d, const void* h, const void* w, const void* bias,
                                       const void* targets, const void* lse, const void* dloss, void* dh, void* dw,
                                       void* dbias, void* workspace, size_t ws_bytes, void* hip_stream) {
  LossArgs a;
  if (int rc = loss_args(d, &a)) return rc;
  if (!dh && !dw && !dbias) return WINO_OK;
  const size_t item = size_of(d->type);
  if (a.rows != 0) {
    const void* given[] = {h, w, targets, lse, dloss};
    const char* names[] = {"h", "w", "targets", "lse", "dloss"};
    const size_t sizes[] = {item, item, 8, 4, 4};
    for (int i = 0; i < 5; ++i) {
      if (int rc = present(given[i], names[i])) return rc;
      if (int rc = on_element(given[i], sizes[i], names[i])) return rc;
    }
  }
  if (int rc = on_element(bias, 4, "bias")) return rc;
  if (int rc = on_element(dh, item, "dh")) return rc;
  if (int rc = on_element(dw, item, "dw")) return rc;
  if (int rc = on_element(dbias, 4, "dbias")) return rc;
  if (a.rows != 0)
    if (int rc = room(workspace, ws_bytes, loss_layout(a, true).bytes)) return rc;
  return failed(launch_loss_backward(a, h, w, (const float*)bias, (const int64_t*)targets, (const float*)lse,
                                     (const float*)dloss, dh, dw, (float*)dbias, (char*)workspace,
                                     (hipStream_t)hip_stream), "cross entropy backward launch");
}

int wino_orthogonalise_workspace_bytes(const wino_orthogonalise_desc_t* d, size_t* bytes) {
  UpdateArgs a;
  if (int rc = update_args(d, &a)) return rc;
  if (!bytes) return refuse(WINO_EINVAL, "%s", "null bytes");
  *bytes = update_layout(a).bytes;
  return WINO_OK;
}

int wino_orthogonalise(const wino_orthogonalise_desc_t* d, const void* g, void* o, void* workspace, size_t ws_bytes,
                       void* hip_stream) {
  UpdateArgs a;
  if (int rc = update_args(d, &a)) return rc;
  if (a.batch == 0 || a.rows == 0 || a.cols == 0) return WINO_OK;
  if (int rc = present(g, "g")) return rc;
  if (int rc = present(o, "o")) return rc;
  if (int rc = on_element(g, size_of(d->g_type), "g")) return rc;
  if (int rc = on_element(o, size_of(d->o_type), "o")) return rc;
  if (int rc = room(workspace, ws_bytes, update_layout(a).bytes)) return rc;
  return failed(launch_update(a, g, o, (char*)workspace, (hipStream_t)hip_stream), "orthogonalise launch");
}

}  // extern "C"
