// Entry points of the operators around the training step: argument checks, and what the launchers need.  Host code only;
// nothing here allocates device memory, synchronises or keeps state between calls.
#include <cmath>
#include <initializer_list>

#include "decoder.h"
#include "train_ops.h"

static_assert(SECO_NORM_BLOCKS == DEC_GAIN_BLOCKS, "the training step adds up the shares of either norm");

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
// whether the rows of d_x and of another tensor share memory, or may
bool overlap(const layer_norm_desc* d, const void* d_x, const void* other, int64_t stride) {
  const uintptr_t e = (uintptr_t)elem(d->dtype), a = reinterpret_cast<uintptr_t>(d_x), b = reinterpret_cast<uintptr_t>(other);
  return a < b + (uintptr_t)((d->rows - 1) * stride + d->d) * e && b < a + (uintptr_t)((d->rows - 1) * d->out_stride + d->d) * e;
}
bool rows_apart(const layer_norm_desc* d, int64_t stride) { return d->rows < 2 || stride >= d->d; }

// ---- AdamW
bool fraction(double b) { return b >= 0.0 && b < 1.0; }
int check_adamw(const adamw_desc* d, const adamw_tensor& t) {
  if (t.n < 0) return SECO_ERR_SHAPE;
  if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.f) return SECO_ERR_RANGE;
  if (!is_dtype(t.param_dtype) || !is_dtype(t.grad_dtype) || (t.master && t.param_dtype != SECO_BF16)) return SECO_ERR_DTYPE;
  if (t.n > (int64_t)1 << 40) return SECO_ERR_TOO_LARGE;
  if (t.n == 0) return SECO_OK;
  const bool eight = d->state_bits == 8;
  if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return SECO_ERR_NULL;
  const int state = eight ? 1 : 4;
  if (!aligned(t.param, elem(t.param_dtype)) || !aligned(t.grad, elem(t.grad_dtype)) || !aligned(t.m, state) || !aligned(t.v, state) ||
      !aligned(t.master, 4) || (eight && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
    return SECO_ERR_ALIGN;
  return SECO_OK;
}
int kind_of(const adamw_desc* d, const adamw_tensor& t) {
  return (t.param_dtype == SECO_BF16 ? kAdamParamBf16 : 0) | (t.grad_dtype == SECO_BF16 ? kAdamGradBf16 : 0) | (t.master ? kAdamMaster : 0) |
         (d->state_bits == 8 ? kAdam8 : 0);
}

// ---- rotary positions with several axes
int check_rope_axes(const seco_desc* d, const rope_axes* x, const int64_t* positions, const int64_t* pos_stride) {
  if (!d || !x || !positions || !pos_stride) return SECO_ERR_NULL;
  if (!is_dtype(d->dtype)) return SECO_ERR_DTYPE;
  if (d->batch < 1 || d->chunk_len < 1 || d->head_dim < 1 || d->q_start < 0) return SECO_ERR_SHAPE;
  if (d->head_dim % 8 != 0 || d->head_dim > 2 * kRopeMaxPairs) return SECO_ERR_HEAD_DIM;
  if (d->batch > 65535 || d->chunk_len > 1 << 27 || (int64_t)d->q_start + d->chunk_len > (int64_t)1 << 30) return SECO_ERR_TOO_LARGE;
  if (x->n_axes < 1 || x->n_axes > SECO_ROPE_MAX_AXES || !std::isfinite(x->base) || !(x->base > 1.f)) return SECO_ERR_RANGE;
  int64_t sum = 0;
  for (int i = 0; i < x->n_axes; ++i) {
    if (x->sections[i] < 0) return SECO_ERR_RANGE;
    sum += x->sections[i];
  }
  if (sum != d->head_dim / 2) return SECO_ERR_RANGE;
  if (!aligned(positions, 8)) return SECO_ERR_ALIGN;
  for (int i = 0; i < 3; ++i) {
    if (pos_stride[i] < 0) return SECO_ERR_SHAPE;
    if (pos_stride[i] > (int64_t)1 << 40) return SECO_ERR_TOO_LARGE;
  }
  return SECO_OK;
}
// frequencies and axes of the pairs, positions
void fill_rope(RopeAxesArgs& a, const seco_desc* d, const rope_axes* x, const int64_t* positions, const int64_t* pos_stride) {
  const int pairs = d->head_dim / 2;
  int left[SECO_ROPE_MAX_AXES], seen[SECO_ROPE_MAX_AXES] = {};
  // base^(-k / n) as a product of powers for the bits of k (an exponential for every pair was a third of a short call's host time)
  double power[SECO_ROPE_MAX_AXES][7];
  const double log2_base = std::log2((double)x->base);
  for (int i = 0; i < x->n_axes; ++i) {
    left[i] = x->sections[i];
    const int n = x->own_frequencies ? x->sections[i] : pairs;
    if (i == 0 || x->own_frequencies)
      for (int j = 0; j < 7 && 1 << j < n; ++j) power[i][j] = std::exp2(-(double)(1 << j) / n * log2_base);
  }
  for (int i = 0, axis = 0; i < pairs; ++i) {
    while (left[axis] == 0) axis = axis + 1 == x->n_axes ? 0 : axis + 1;   // (some axis lacks pairs: they add up)
    a.axis[i] = (uint8_t)axis;
    const double* of = power[x->own_frequencies ? axis : 0];
    double f = 1.0;
    for (int k = x->own_frequencies ? seen[axis] : i, j = 0; k; k >>= 1, ++j)
      if (k & 1) f *= of[j];
    a.frequency[i] = f;
    ++seen[axis];
    --left[axis];
    if (x->interleaved) axis = axis + 1 == x->n_axes ? 0 : axis + 1;
  }
  a.positions = positions;
  for (int i = 0; i < 3; ++i) a.ps[i] = pos_stride[i];
  a.B = d->batch;
  a.C = d->chunk_len;
  a.D = d->head_dim;
  a.n_axes = x->n_axes;
  a.scale = 1.f;
}
// one tensor pair; rows from in_row, out_row on.  Rows start on 16-byte boundaries, as everywhere.
int set_part(RopePart& p, const seco_desc* d, const void* in, void* out, int heads, const int64_t* is, const int64_t* os, int in_elem,
             int out_elem, int64_t in_row, int64_t out_row) {
  if ((in == nullptr) != (out == nullptr)) return SECO_ERR_NULL;
  if (!in) return SECO_OK;
  if (heads < 1) return SECO_ERR_SHAPE;
  if (heads > 65535) return SECO_ERR_TOO_LARGE;
  for (int i = 0; i < 3; ++i) {
    const int64_t most = (int64_t)1 << (i == 2 ? 30 : 40);          // (rows start at row * stride, row up to 2^30)
    if (is[i] > most || os[i] > most) return SECO_ERR_TOO_LARGE;
    if (is[i] < 0 || is[i] * in_elem % 16 || os[i] < 0 || os[i] * out_elem % 16) return SECO_ERR_ALIGN;
  }
  if (is[2] < d->head_dim || os[2] < d->head_dim) return SECO_ERR_ALIGN;
  if (!aligned(in, 16) || !aligned(out, 16)) return SECO_ERR_ALIGN;
  p.in = static_cast<const char*>(in) + in_row * is[2] * in_elem;
  p.out = static_cast<char*>(out) + out_row * os[2] * out_elem;
  for (int i = 0; i < 3; ++i) {
    p.is[i] = is[i];
    p.os[i] = os[i];
  }
  p.heads = heads;
  return SECO_OK;
}

}  // namespace
}  // namespace seco

using namespace seco;

extern "C" int rope_rotate_axes(const seco_desc* desc, const rope_axes* axes, int32_t n_heads, const void* x_in, void* x_out,
                                const int64_t* positions, const int64_t* pos_stride, int32_t inverse, void* hip_stream) {
  int rc = check_rope_axes(desc, axes, positions, pos_stride);
  if (rc) return rc;
  if (!x_in || !x_out) return SECO_ERR_NULL;
  RopeAxesArgs a{};
  const int e = elem(desc->dtype);
  if ((rc = set_part(a.q, desc, x_in, x_out, n_heads, desc->q_stride, desc->o_stride, e, e, 0, 0))) return rc;
  fill_rope(a, desc, axes, positions, pos_stride);
  return launch_rope_axes(a, desc->dtype == SECO_BF16, false, inverse != 0, static_cast<hipStream_t>(hip_stream));
}

extern "C" int rope_append_axes(const seco_desc* desc, const rope_axes* axes, const void* q, void* q_out, const void* k_new,
                                const void* v_new, void* k_cache, void* v_cache, const int64_t* positions, const int64_t* pos_stride,
                                void* hip_stream) {
  int rc = check_rope_axes(desc, axes, positions, pos_stride);
  if (rc) return rc;
  RopeAxesArgs a{};
  const int e = elem(desc->dtype);
  const int64_t row = desc->q_start;
  if ((rc = set_part(a.q, desc, q, q_out, desc->n_q_heads, desc->q_stride, desc->o_stride, e, e, 0, 0))) return rc;
  if ((rc = set_part(a.k, desc, k_new, k_cache, desc->n_kv_heads, desc->g_stride, desc->kv_stride, e, e, 0, row))) return rc;
  if ((rc = set_part(a.v, desc, v_new, v_cache, desc->n_kv_heads, desc->g_stride, desc->kv_stride, e, e, 0, row))) return rc;
  if (!q && !k_new && !v_new) return SECO_OK;
  fill_rope(a, desc, axes, positions, pos_stride);
  return launch_rope_axes(a, desc->dtype == SECO_BF16, false, false, static_cast<hipStream_t>(hip_stream));
}

extern "C" int rope_readout_axes(const seco_desc* desc, const rope_axes* axes, const void* d_q, void* d_q_out, const float* gk,
                                 const float* gv, void* d_k_new, void* d_v_new, float scaler, const int64_t* positions,
                                 const int64_t* pos_stride, void* hip_stream) {
  int rc = check_rope_axes(desc, axes, positions, pos_stride);
  if (rc) return rc;
  if (!std::isfinite(scaler)) return SECO_ERR_RANGE;
  RopeAxesArgs a{};
  const int e = elem(desc->dtype);
  const int64_t row = desc->q_start;
  if ((rc = set_part(a.q, desc, d_q, d_q_out, desc->n_q_heads, desc->q_stride, desc->o_stride, e, e, 0, 0))) return rc;
  if ((rc = set_part(a.k, desc, gk, d_k_new, desc->n_kv_heads, desc->g_stride, desc->kv_stride, 4, e, row, 0))) return rc;
  if ((rc = set_part(a.v, desc, gv, d_v_new, desc->n_kv_heads, desc->g_stride, desc->kv_stride, 4, e, row, 0))) return rc;
  if (!d_q && !gk && !gv) return SECO_OK;
  fill_rope(a, desc, axes, positions, pos_stride);
  a.scale = scaler;
  return launch_rope_axes(a, desc->dtype == SECO_BF16, desc->dtype == SECO_BF16, true, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t layer_norm_workspace_bytes(const layer_norm_desc* desc) {
  if (check_norm(desc)) return (size_t)-1;
  if (norm_few(desc->rows, desc->d)) return 0;
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
  const bool few = sums && norm_few(desc->rows, desc->d);
  if (sums && !few && (!ws || !aligned(ws, 16) || ws_bytes < layer_norm_workspace_bytes(desc))) return SECO_ERR_WORKSPACE;
  if (desc->rows == 0 && !sums) return SECO_OK;
  NormArgs a = norm_args(desc);
  a.x = x;
  a.r = d_in;
  a.gain = gain;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dy = d_y;
  a.out = d_x;
  a.blocks = a.part_rows = norm_blocks(desc->rows, desc->d, desc->dtype);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (few) {                                     // (d_x in the place of what the sums are made of: the sums first)
    a.d_gain = d_gain;
    a.d_bias = d_bias;
    const bool apart = !overlap(desc, d_x, x, desc->x_stride) && !overlap(desc, d_x, d_y, desc->y_stride);
    rc = launch_norm_bwd_few(a, apart, true, s);
    return rc || apart ? rc : launch_norm_bwd_few(a, true, false, s);
  }
  a.parts = sums ? static_cast<float*>(ws) : nullptr;
  rc = launch_norm_bwd(a, s);
  if (rc || !sums) return rc;
  return launch_norm_sums(a.parts, a.blocks, a.d, d_gain, d_bias, a.gain_f32, s);
}

extern "C" int adamw_step(const adamw_desc* desc, const adamw_tensor* tensors_host, int32_t n_tensors, int64_t* step, void* hip_stream) {
  if (!desc || !step || (n_tensors > 0 && !tensors_host)) return SECO_ERR_NULL;
  if (n_tensors < 0) return SECO_ERR_SHAPE;
  if (desc->state_bits != 8 && desc->state_bits != 32) return SECO_ERR_DTYPE;
  if (!std::isfinite(desc->lr) || desc->lr < 0.0 || !fraction(desc->beta1) || !fraction(desc->beta2) || !std::isfinite(desc->eps) ||
      desc->eps < 0.0)
    return SECO_ERR_RANGE;
  if (!aligned(step, 8) || !aligned(desc->lr_device, 4) || !aligned(desc->grad_scale_device, 4)) return SECO_ERR_ALIGN;
  unsigned kinds = 0;                            // that there are
  for (int32_t i = 0; i < n_tensors; ++i) {
    if (const int rc = check_adamw(desc, tensors_host[i])) return rc;
    kinds |= 1u << kind_of(desc, tensors_host[i]);
  }
  AdamArgs a{};
  a.lr = desc->lr;
  a.beta1 = desc->beta1;
  a.beta2 = desc->beta2;
  a.eps = (float)desc->eps;
  a.lr_at = desc->lr_device;
  a.grad_scale = desc->grad_scale_device;
  a.step = step;
  hipStream_t hs = static_cast<hipStream_t>(hip_stream);
  const int64_t span = adam_span(desc->state_bits == 8);
  int64_t all = 0;
  for (int32_t i = 0; i < n_tensors; ++i) all += (tensors_host[i].n + span - 1) / span;
  if (all > kAdamCounting) {
    if (const int rc = launch_adamw_count(step, hs)) return rc;
    a.counted = 1;
  }
  // Tensors of one kind share launches; one that is full waits for the next tensor, so that the last launch is known as such.
  int pending = 0, rc = SECO_OK;
  for (int kind = 0; kind < 16 && !rc; ++kind)
    for (int32_t i = 0; kinds >> kind & 1 && i < n_tensors && !rc; ++i) {
      const adamw_tensor& t = tensors_host[i];
      if (t.n == 0 || kind_of(desc, t) != kind) continue;
      const uint32_t spans = (uint32_t)((t.n + span - 1) / span);      // at most 2^30
      if (a.count == kAdamTensors || (a.count && (pending != kind || a.spans + spans > (uint32_t)1 << 31))) {
        rc = launch_adamw(pending, a, hs);
        a.count = 0;
        a.spans = 0;
      }
      pending = kind;
      a.e[a.count++] = AdamEntry{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.master, a.spans, a.spans + spans - 1,
                                 (int)(t.n - (int64_t)(spans - 1) * span), t.weight_decay};
      a.spans += spans;
    }
  if (rc || (a.counted && !a.count)) return rc;
  a.last = !a.counted;
  return launch_adamw(pending, a, hs);
}

// ---- layer norm in the training step (decoder.h): contiguous rows, gain and bias of their type
namespace {
NormArgs step_norm(int dtype, const void* gain, const void* bias, float eps, int64_t rows, int64_t d) {
  NormArgs a{};
  a.rows = rows;
  a.d = a.xs = a.rs = a.os = a.ys = d;
  a.dtype = dtype;
  a.gain_f32 = dtype == SECO_F32;
  a.gain = gain;
  a.bias = bias;
  a.eps = eps;
  return a;
}
bool step_sizes(int dtype, int64_t rows, int64_t d) { return is_dtype(dtype) && rows >= 0 && rows < (int64_t)1 << 31 && d >= 1 && d <= (int64_t)1 << 30; }
}  // namespace

extern "C" int dec_add_layer_norm(int dtype, const void* x, const void* y, const void* gain, const void* bias, float eps, void* x_out, void* h,
                                  float* mean, float* rstd, int64_t rows, int64_t d, void* stream) {
  if (!step_sizes(dtype, rows, d)) return SECO_ERR_SHAPE;
  if (rows == 0) return SECO_OK;
  NormArgs a = step_norm(dtype, gain, bias, eps, rows, d);
  a.x = x;
  a.r = y;
  a.out = y ? x_out : nullptr;
  a.y = h;
  a.mean = mean;
  a.rstd = rstd;
  return launch_norm_fwd(a, static_cast<hipStream_t>(stream));
}

extern "C" int dec_embed_layer_norm(int dtype, const void* table, const int64_t* token, const void* gain, const void* bias, float eps, void* x_out,
                                    void* h, float* mean, float* rstd, int64_t rows, int64_t d, int64_t v, float* outside, void* stream) {
  if (!step_sizes(dtype, rows, d) || v < 1) return SECO_ERR_SHAPE;
  if (rows == 0) return SECO_OK;
  NormArgs a = step_norm(dtype, gain, bias, eps, rows, d);
  a.x = table;
  a.token = token;
  a.table = v;
  a.outside = outside;
  a.out = x_out;
  a.y = h;
  a.mean = mean;
  a.rstd = rstd;
  return launch_norm_fwd(a, static_cast<hipStream_t>(stream));
}

extern "C" int dec_layer_norm_bwd(int dtype, const void* x, const void* gain, const float* mean, const float* rstd, const void* d_h,
                                  const void* d_in, void* d_x, float* parts, int64_t rows, int64_t d, void* stream) {
  if (!step_sizes(dtype, rows, d)) return SECO_ERR_SHAPE;
  if (rows == 0) return SECO_OK;
  NormArgs a = step_norm(dtype, gain, nullptr, 0.f, rows, d);
  a.x = x;
  a.r = d_in;
  a.dy = d_h;
  a.out = d_x;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.part_rows = SECO_NORM_BLOCKS;
  a.accumulate = 1;
  if (norm_few(rows, d)) {                // (into the first share; d_x overwrites neither x nor d_h here)
    a.d_gain = parts;
    a.d_bias = parts + SECO_NORM_BLOCKS * d;
    return launch_norm_bwd_few(a, true, true, static_cast<hipStream_t>(stream));
  }
  a.parts = parts;
  a.blocks = norm_blocks(rows, d, dtype);
  return launch_norm_bwd(a, static_cast<hipStream_t>(stream));
}
