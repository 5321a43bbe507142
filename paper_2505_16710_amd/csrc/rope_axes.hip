// Rotary positions with several axes (time, height, width): the pair (x[i], x[i + D/2]) of a row turns by the row's position on
// the pair's axis times the pair's frequency.  One launch takes a layer's queries (turned), its keys (turned, to or
// from the cache) and its values (copied or converted).
//
// Bound by memory.  Angles, sines and products are fp64 as in the rotation with one axis (rope.h), one rounding of the
// result: of a frame at position 30000 an fp32 angle would be off by 1e-3.  Sines depend on the row and the pair only: a thread
// takes kPairs consecutive pairs of one row (both halves) for kHeads heads.  All of a thread's loads are issued in front of the
// arithmetic, the row's positions on every axis among them, so that no load waits for another.  Four pairs and four heads:
// with eight pairs (16 bytes of bf16 to an access) a row's sines are a longer chain for fewer threads, one token of 32/8 heads
// 4.1 us instead of 3.2, 16384 rows 92 instead of 87; with two heads 2048 rows 13.1 instead of 11.8, with eight 512 the same.
#include "rope.h"
#include "row_tiles.h"
#include "train_ops.h"

namespace seco {
namespace {

constexpr int kThreads = 256, kHeads = 4, kPairs = 4, kSlab = 65535;

template <typename TIn, typename TOut, bool INV>
__device__ __forceinline__ void heads_of(const RopeAxesArgs& a, const RopePart& p, int group, int b, int row, int pair, bool plain, float scale) {
  constexpr int V = kPairs;
  const int h0 = group * kHeads, heads = min(kHeads, p.heads - h0), half = a.D / 2;
  const TIn* in = static_cast<const TIn*>(p.in) + b * p.is[0] + h0 * p.is[1] + (int64_t)row * p.is[2] + pair;
  TOut* out = static_cast<TOut*>(p.out) + b * p.os[0] + h0 * p.os[1] + (int64_t)row * p.os[2] + pair;
  Pack<TIn, V> lo[kHeads], hi[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const TIn* at = in + (h < heads ? h : 0) * p.is[1];
    lo[h] = Pack<TIn, V>::at(at);
    hi[h] = Pack<TIn, V>::at(at + half);
  }
  if (plain) {
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < heads) {
        float f[V];
        lo[h].get(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] *= scale;
        Pack<TOut, V>::of(f).to(out + h * p.os[1]);
        hi[h].get(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] *= scale;
        Pack<TOut, V>::of(f).to(out + h * p.os[1] + half);
      }
    return;
  }
  double at[4];
  const int64_t* pos = a.positions + b * a.ps[1] + (int64_t)row * a.ps[2];
#pragma unroll
  for (int x = 0; x < 4; ++x) at[x] = (double)pos[(x < a.n_axes ? x : 0) * a.ps[0]];
  double sn[V], cs[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int x = a.axis[pair + j];
    const double p01 = x & 1 ? at[1] : at[0], p23 = x & 1 ? at[3] : at[2];
    sincos_f64((x & 2 ? p23 : p01) * a.frequency[pair + j], sn[j], cs[j]);
    sn[j] *= INV ? -(double)scale : (double)scale;
    cs[j] *= (double)scale;
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h)
    if (h < heads) {
      float f[V], g[V];
      lo[h].get(f);
      hi[h].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) rope_pair(f[j], g[j], sn[j], cs[j]);
      Pack<TOut, V>::of(f).to(out + h * p.os[1]);
      Pack<TOut, V>::of(g).to(out + h * p.os[1] + half);
    }
}

// blockIdx.x: head groups of q, then of k, then of v, so that neighbours share rows (16384 rows of 32/8 heads 76 us, with the rows
// along x 87); y: rows, 65535 workgroups of them to a slab; z: slabs of a batch, batches
template <typename T, typename TIn, bool INV>
__global__ __launch_bounds__(kThreads) void rope_axes_kernel(RopeAxesArgs a) {
  const int per = a.D / 2 / kPairs, rows = kThreads / per, lr = threadIdx.x / per, row = ((int)(blockIdx.z % a.slabs) * kSlab + (int)blockIdx.y) * rows + lr, pair = (threadIdx.x - lr * per) * kPairs;
  if (lr >= rows || row >= a.C) return;
  const int nq = (a.q.heads + kHeads - 1) / kHeads, nk = (a.k.heads + kHeads - 1) / kHeads, y = blockIdx.x, b = blockIdx.z / a.slabs;
  if (y < nq) heads_of<T, T, INV>(a, a.q, y, b, row, pair, false, 1.f);
  else if (y < nq + nk) heads_of<TIn, T, INV>(a, a.k, y - nq, b, row, pair, false, a.scale);
  else heads_of<TIn, T, INV>(a, a.v, y - nq - nk, b, row, pair, true, a.scale);
}

int row_blocks(const RopeAxesArgs& a) {
  const int rows = kThreads / (a.D / 2 / kPairs);
  return (a.C + rows - 1) / rows;
}
template <typename T, typename TIn, bool INV> void launch(const RopeAxesArgs& a, hipStream_t s) {
  const int n = row_blocks(a);
  auto groups = [](int heads) { return (heads + kHeads - 1) / kHeads; };
  const dim3 grid((unsigned)(groups(a.q.heads) + groups(a.k.heads) + groups(a.v.heads)), (unsigned)(n < kSlab ? n : kSlab), (unsigned)(a.B * a.slabs));
  hipLaunchKernelGGL((rope_axes_kernel<T, TIn, INV>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

int launch_rope_axes(const RopeAxesArgs& args, bool bf16, bool wide_in, bool inverse, hipStream_t s) {
  RopeAxesArgs a = args;
  a.slabs = (row_blocks(a) + kSlab - 1) / kSlab;
  if ((int64_t)a.B * a.slabs > 65535) return SECO_ERR_TOO_LARGE;
  if (!bf16) inverse ? launch<float, float, true>(a, s) : launch<float, float, false>(a, s);
  else if (wide_in) launch<__bf16, float, true>(a, s);
  else inverse ? launch<__bf16, __bf16, true>(a, s) : launch<__bf16, __bf16, false>(a, s);
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

}  // namespace seco
