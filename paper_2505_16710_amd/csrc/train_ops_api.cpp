// Entry points of the operators around the training step: argument checks, and what the launchers need.  Host code only;
// nothing here allocates device memory, synchronises or keeps state between calls.
#include <cmath>

#include "train_ops.h"

namespace seco {
namespace {

bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
int elem(int dtype) { return dtype == SECO_BF16 ? 2 : 4; }
bool is_dtype(int dtype) { return dtype == SECO_F32 || dtype == SECO_BF16; }

// ---- layer norm
int check_norm(const layer_norm_desc* d) {
  if (!d) return SECO_ERR_NULL;
  if (!is_dtype(d->dtype) || (d->gain_dtype != d->dtype && d->gain_dtype != SECO_F32)) return SECO_ERR_DTYPE;
  if (d->rows < 0 || d->d < 1) return SECO_ERR_SHAPE;
  if (!std::isfinite(d->eps) || d->eps < 0.f) return SECO_ERR_RANGE;
  if (d->d > (int64_t)1 << 30 || d->rows > (int64_t)1 << 31) return SECO_ERR_TOO_LARGE;
  for (int64_t s : {d->x_stride, d->residual_stride, d->out_stride, d->y_stride}) {
    if (s < 0) return SECO_ERR_SHAPE;
    if (s > (int64_t)1 << 31) return SECO_ERR_TOO_LARGE;
  }
  return SECO_OK;
}
NormArgs norm_args(const layer_norm_desc* d) {
  NormArgs a{};
  a.rows = d->rows;
  a.d = d->d;
  a.xs = d->x_stride;
  a.rs = d->residual_stride;
  a.os = d->out_stride;
  a.ys = d->y_stride;
  a.eps = d->eps;
  a.dtype = d->dtype;
  a.gain_f32 = d->gain_dtype == SECO_F32;
  return a;
}
bool rows_apart(const layer_norm_desc* d, int64_t stride) { return d->rows < 2 || stride >= d->d; }

}  // namespace
}  // namespace seco

using namespace seco;

extern "C" size_t layer_norm_workspace_bytes(const layer_norm_desc* desc) {
  if (check_norm(desc)) return (size_t)-1;
  return (size_t)2 * norm_blocks(desc->rows, desc->d, desc->dtype) * desc->d * sizeof(float);
}

extern "C" int layer_norm_fwd(const layer_norm_desc* desc, const void* x, const void* residual, const void* gain, const void* bias,
                              void* x_out, void* y, float* mean, float* rstd, void* hip_stream) {
  int rc = check_norm(desc);
  if (rc) return rc;
  if (!x || !y || !mean || !rstd || (residual != nullptr) != (x_out != nullptr)) return SECO_ERR_NULL;
  const int e = elem(desc->dtype), ge = elem(desc->gain_dtype);
  for (const void* p : {x, residual, (const void*)x_out, (const void*)y})
    if (!aligned(p, e)) return SECO_ERR_ALIGN;
  if (!aligned(gain, ge) || !aligned(bias, ge) || !aligned(mean, 4) || !aligned(rstd, 4)) return SECO_ERR_ALIGN;
  if (!rows_apart(desc, desc->y_stride) || (x_out && !rows_apart(desc, desc->out_stride))) return SECO_ERR_SHAPE;
  if (desc->rows == 0) return SECO_OK;
  NormArgs a = norm_args(desc);
  a.x = x;
  a.r = residual;
  a.gain = gain;
  a.bias = bias;
  a.out = x_out;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  return launch_norm_fwd(a, static_cast<hipStream_t>(hip_stream));
}

extern "C" int layer_norm_bwd(const layer_norm_desc* desc, const void* x, const void* gain, const float* mean, const float* rstd,
                              const void* d_y, const void* d_in, void* d_x, void* d_gain, void* d_bias, void* ws, size_t ws_bytes,
                              void* hip_stream) {
  int rc = check_norm(desc);
  if (rc) return rc;
  if (!x || !mean || !rstd || !d_y || !d_x) return SECO_ERR_NULL;
  const int e = elem(desc->dtype), ge = elem(desc->gain_dtype);
  for (const void* p : {x, d_y, d_in, (const void*)d_x})
    if (!aligned(p, e)) return SECO_ERR_ALIGN;
  if (!aligned(gain, ge) || !aligned(d_gain, ge) || !aligned(d_bias, ge) || !aligned(mean, 4) || !aligned(rstd, 4)) return SECO_ERR_ALIGN;
  if (!rows_apart(desc, desc->out_stride)) return SECO_ERR_SHAPE;
  const bool sums = d_gain || d_bias;
  if (sums && (!ws || !aligned(ws, 16) || ws_bytes < layer_norm_workspace_bytes(desc))) return SECO_ERR_WORKSPACE;
  if (desc->rows == 0 && !sums) return SECO_OK;
  NormArgs a = norm_args(desc);
  a.x = x;
  a.r = d_in;
  a.gain = gain;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dy = d_y;
  a.out = d_x;
  a.parts = sums ? static_cast<float*>(ws) : nullptr;
  a.blocks = norm_blocks(desc->rows, desc->d, desc->dtype);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  rc = launch_norm_bwd(a, s);
  if (rc || !sums) return rc;
  return launch_norm_sums(a.parts, a.blocks, a.d, d_gain, d_bias, a.gain_f32, s);
}
