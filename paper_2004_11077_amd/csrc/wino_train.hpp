// Launchers of the operators of a training step (wino_norm.hip, wino_loss.hip, wino_update.hip)
// behind the entry points in wino_train.cpp.  Not part of the public boundary.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace wino {

inline size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// ---- layer norm ------------------------------------------------------------------------------
struct NormArgs {
  long rows;
  int channels, x_type, y_type, g_type;
  float eps;
  double s, inv_s, inv_c; // s_y, 1 / s_y, 1 / channels
  long x_stride, y_stride, dy_stride, dx_stride;
};
hipError_t launch_norm(const NormArgs& a, const void* x, const float* gamma, const float* beta, void* y,
                       float* mean, float* rstd, hipStream_t st);
// Work groups of the backward kernel, each with one partial sum of dgamma and of dbeta.
int norm_parts(long rows, int channels);
hipError_t launch_norm_backward(const NormArgs& a, const void* dy, const void* x, const float* gamma,
                                const float* mean, const float* rstd, void* dx, float* dgamma,
                                float* dbeta, float* parts, hipStream_t st);

// ---- linear cross entropy --------------------------------------------------------------------
struct LossArgs {
  int rows, features, classes;
  int bf16;               // operands and gradients: 0 fp32, 1 bf16
  long h_stride, w_stride;
  long ignore_index;
  int piece;              // classes per piece (0: chosen here)
};
// Regions of the workspace, bytes from its start; `bytes` in all.
struct LossLayout {
  int piece, dp;          // classes per piece; features rounded up to whole lines
  int side, dh_side;      // tiles of dl's and dh's products
  int splits;             // ranges of the classes of a piece in dh's product
  int dw_splits;          // ranges of the rows in dW's product
  int two;                // bf16: dl on two values
  size_t numbers, w, h, parts, target, unit_w, unit_h, dl, rest, dh, dw, dbias, bytes;
};
hipError_t launch_loss(const LossArgs& a, const void* h, const void* w, const float* bias,
                       const int64_t* target, float* loss, float* lse, char* ws, hipStream_t st);
hipError_t launch_loss_backward(const LossArgs& a, const void* h, const void* w, const float* bias,
                                const int64_t* target, const float* lse, const float* dloss, void* dh,
                                void* dw, float* dbias, char* ws, hipStream_t st);

// ---- orthogonalised updates ------------------------------------------------------------------
struct UpdateArgs {
  int batch, rows, cols, g_bf16, o_bf16, steps;
  float a, b, c, eps, scale;
  long g_batch, g_stride, o_batch, o_stride;
};
struct UpdateLayout {
  int r, c, rp, cp;           // r <= c: the smaller and the larger side; rounded up to whole lines
  int side, splits;           // tiles and ranges of k of A's product
  size_t norms, x, x2, gram, poly, parts, bytes;
};
hipError_t launch_update(const UpdateArgs& a, const void* g, void* o, char* ws, hipStream_t st);

}  // namespace wino
