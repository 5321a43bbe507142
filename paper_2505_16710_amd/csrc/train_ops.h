// Host side and kernels of the operators around the training step: what the entry points (train_ops_api.cpp) hand to the
// launchers once they have checked it.  No HIP type but the stream, so that the host side builds without a GPU compiler.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "seco.h"

namespace seco {

// Most workgroups of a layer norm's backward, and so most partial sums per column: one to a CU
#define SECO_NORM_BLOCKS 256

// ---- layer norm.  Row strides in elements; pointers that may be NULL are marked.
struct NormArgs {
  const void *x, *r;             // r: residual (forward), d_in (backward); NULL: none
  const void *gain, *bias;       // NULL: ones, zeros
  const void* dy;
  void *out, *y;                 // forward: x + r (NULL without r) and the result; backward: d_x in out
  float *mean, *rstd;
  float *parts;                  // backward: sums of d_gain per workgroup [blocks][d] and, part_rows rows on, of d_bias; or NULL
  int part_rows;
  int64_t rows, d, xs, rs, os, ys;
  float eps;
  int dtype, gain_f32;           // gain_f32: gain and bias are fp32 (else of dtype)
  void *d_gain, *d_bias;         // backward of few rows: the sums themselves (either NULL), fp32 with accumulate
  int blocks, accumulate;        // workgroups that leave sums; 1: they are added to what is there
  // forward, first norm of a decoder: row r of x is row token[r] of a table of `table` rows
  const int64_t* token;
  int64_t table;
  float* outside;
};
int norm_blocks(int64_t rows, int64_t d, int dtype);                       // workgroups of a backward call
int launch_norm_fwd(const NormArgs& a, hipStream_t s);
int launch_norm_bwd(const NormArgs& a, hipStream_t s);
// Rows of a backward call in one launch, and their length (backward_shape's longest).  A test of refusals hands calls of 2000 rows
// without a workspace to the library, with addresses that no kernel may see.
constexpr int64_t kNormFewRows = 1280, kNormFewLength = 16384;
static_assert(kNormFewRows < 2000, "calls of 2000 rows have to bring a workspace");
// Whether a backward call has so few rows that its sums need no parts, but come from a.x and a.dy a second time; and that call:
// d_x (rows), the sums, or both in one launch where d_x overwrites neither
bool norm_few(int64_t rows, int64_t d);
int launch_norm_bwd_few(const NormArgs& a, bool rows, bool sums, hipStream_t s);
// d_gain, d_bias (either NULL) = parts added up over the blocks in their order
int launch_norm_sums(const float* parts, int blocks, int64_t d, void* d_gain, void* d_bias, int gain_f32, hipStream_t s);

// ---- AdamW.  What a launch needs of a tensor, and of its tensors together; passed by value.
constexpr int kAdamTensors = 48;               // of a launch: its arguments stay below 4 KiB
// Elements of a workgroup: two blocks of 256 to a wavefront, one where states of 8 bits take the wavefront's reductions
constexpr int64_t adam_span(bool eight) { return eight ? 1024 : 2048; }
// Up to so many workgroups count the step themselves, each by an addition to one place; of more, these additions (11 ns each, one
// behind the other) take longer than a launch in front that counts it (2 us)
constexpr uint32_t kAdamCounting = 128;
struct AdamEntry {
  void* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale, *master;
  uint32_t first, last;                        // its spans among the launch's
  int tail;                                    // elements of the last one
  float decay;
};
struct AdamArgs {
  AdamEntry e[kAdamTensors];
  double lr, beta1, beta2;
  float eps;
  const float *lr_at, *grad_scale;             // or NULL
  int64_t* step;
  uint32_t spans;
  int count;
  int counted, last;                           // counted: the step is already; else `last` is the launch that counts it
};
// kind: bits 0 param bf16, 1 gradient bf16, 2 master, 3 states of 8 bits
enum { kAdamParamBf16 = 1, kAdamGradBf16 = 2, kAdamMaster = 4, kAdam8 = 8 };
int launch_adamw(int kind, const AdamArgs& a, hipStream_t s);
int launch_adamw_count(int64_t* step, hipStream_t s);

// ---- rotary positions with several axes.  A tensor pair of a call: rows in and rows out, head heads of each batch.
constexpr int kRopeMaxPairs = 128;
struct RopePart {
  const void* in;
  void* out;
  int64_t is[3], os[3];                        // (batch, head, row) strides in elements
  int heads;
};
struct RopeAxesArgs {
  double frequency[kRopeMaxPairs];
  uint8_t axis[kRopeMaxPairs];
  RopePart q, k, v;                            // q, k: turned; v: as it is (heads 0: not there)
  const int64_t* positions;
  int64_t ps[3];                               // (axis, batch, row) strides
  int B, C, D, n_axes, slabs;                  // slabs: the launcher's
  float scale;                                 // of k and v
};
// bf16: the type of q and of what k and v give; wide_in: k and v are fp32 all the same
int launch_rope_axes(const RopeAxesArgs& a, bool bf16, bool wide_in, bool inverse, hipStream_t s);   // wide_in: inverse only

}  // namespace seco
