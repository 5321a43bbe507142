// The AdamW update of many tensors in one launch.  Per element, with t = steps taken before + 1 and g the scaled gradient:
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// in fp32; the factors of the step in fp64, once per workgroup.  A bf16 p is rounded from its fp32 master, or from itself.
//
// States of 8 bits: a block of 256 consecutive elements of a tensor holds m and r = sqrt(v) as e4m3 codes in units of the block's
// largest magnitude / 448.  That unit is no power of two, so that the largest element is kept to fp32: a block whose squares all
// decay by b2 = 0.999 a step keeps its codes and follows in its unit, while a single code could not move by so little.  r instead
// of v: its three bits and 18 powers of two of range then hold v over 36.  An r that is not zero is never stored as
// zero (its m / eps would be unbounded), but as at least the smallest code; an infinite one, for which there is no code, as NaN.  The update itself uses m and v before they are rounded.
// What is stored is rounded to fp32 operation by operation: (1 - b) g is added to the product b m in one fused operation, the unit is
// the largest magnitude times the rounded 1 / 448, root and quotient are to the nearest.  A value one step of fp32 off would now and
// then take the neighbouring code, an eighth away, and with it the steps behind.
//
// Bound by memory: 28 bytes per element with fp32 masters and states, 16.06 with states of 8 bits.  A wavefront takes a block at
// a time, 4 elements to a lane, so that a block's largest magnitudes are a reduction over its lanes.
#include "row_tiles.h"
#include "train_ops.h"

#pragma clang fp contract(off)

namespace seco {
namespace {

constexpr int kThreads = 256, kBlockLen = 256;
constexpr float kTop = 448.f, kLeast = 0x1p-9f;      // the largest and the smallest positive e4m3 value

// b^t for t >= 1
__device__ __forceinline__ double power(double b, uint64_t t) {
  double r = 1.0;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

struct Factors {
  float rate, inv_root, lr;
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode(unsigned codes, float unit, float (&f)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo[0] * unit;
  f[1] = lo[1] * unit;
  f[2] = hi[0] * unit;
  f[3] = hi[1] * unit;
}
__device__ __forceinline__ unsigned encode(const float (&f)[4]) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
}
// the largest finite magnitude of a block / 448, in every lane
__device__ __forceinline__ float unit_of(const float (&f)[4]) {
  float top = wave_max(fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3]))));   // (without the NaN)
  if (__builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, top)) == 0x7f800000) {
    top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(f[j]) < INFINITY ? fabsf(f[j]) : 0.f);
    top = wave_max(top);
  }
  return fmaxf(top * (1.f / kTop), 0x1p-126f);
}
// 1 / x and a / x, given 1 / x, to the nearest: one correction of what is a step off at most
__device__ __forceinline__ float reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.f), r, r);
}
__device__ __forceinline__ float quotient(float a, float x, float inv) {
  const float q = a * inv;
  return fmaf(fmaf(-q, x, a), inv, q);
}
// The hardware's root (a step off at most) takes a square below 2^-126 for zero: those are moved up by 2^64 and their roots down
// by 2^-32, both exact.  That takes 1.2 % of the time of 478M elements in 8 bits (1278 -> 1293 us), 0.6 % in 32; a branch around it for
// wavefronts that hold such squares takes 5 %.
__device__ __forceinline__ float root_down(float x) { return x < 0x1p-96f ? 0x1p-32f : 1.f; }
__device__ __forceinline__ float root_up(float x) { return x < 0x1p-96f ? x * 0x1p64f : x; }
__device__ __forceinline__ float near_root(float x) { return __builtin_amdgcn_sqrtf(root_up(x)) * root_down(x); }
// the root to the nearest: of the hardware's and its neighbours one fits
__device__ __forceinline__ float root(float y) {
  const float x = root_up(y), s = __builtin_amdgcn_sqrtf(x);
  const float dn = __builtin_bit_cast(float, __builtin_bit_cast(int, s) - 1), up = __builtin_bit_cast(float, __builtin_bit_cast(int, s) + 1);
  const float r = fmaf(-dn, s, x) <= 0.f ? dn : s;
  return (fmaf(-up, s, x) > 0.f ? up : r) * root_down(y);
}

// What a lane holds of a block
template <typename P, typename G, bool MASTER, int BITS> struct Lane {
  Pack<G, 4> g;
  Pack<float, 4> w;                              // master, or fp32 parameter
  Pack<P, 4> p;
  Pack<float, 4> m, v;
  unsigned mc, vc;
  float mu, vu;
};

// n: elements of the block; FULL: all 256
template <bool FULL, typename T> __device__ __forceinline__ Pack<T, 4> read(const T* p, unsigned c, int n) {
  if constexpr (FULL) return Pack<T, 4>::once(p, c);
  float f[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = (int)c + j < n ? (float)p[c + j] : 0.f;
  return Pack<T, 4>::of(f);
}
template <bool FULL, typename T> __device__ __forceinline__ void write(T* p, unsigned c, int n, const float (&f)[4]) {
  if constexpr (FULL) return Pack<T, 4>::of(f).away(p, c);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if ((int)c + j < n) p[c + j] = (T)f[j];
}
template <bool FULL> __device__ __forceinline__ unsigned read_codes(const void* at, unsigned c, int n) {
  const uint8_t* p = static_cast<const uint8_t*>(at);
  unsigned u = 0;
  if constexpr (FULL) {
    typedef unsigned loose __attribute__((aligned(1)));
    u = __builtin_nontemporal_load(reinterpret_cast<const loose*>(p + c));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)c + j < n) u |= (unsigned)p[c + j] << 8 * j;
  }
  return u;
}
template <bool FULL> __device__ __forceinline__ void write_codes(void* at, unsigned c, int n, unsigned u) {
  uint8_t* p = static_cast<uint8_t*>(at);
  if constexpr (FULL) {
    typedef unsigned loose __attribute__((aligned(1)));
    __builtin_nontemporal_store(u, reinterpret_cast<loose*>(p + c));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)c + j < n) p[c + j] = (uint8_t)(u >> 8 * j);
  }
}

template <typename P, typename G, bool MASTER, int BITS, bool FULL>
__device__ __forceinline__ void fetch(Lane<P, G, MASTER, BITS>& l, const AdamEntry& e, int64_t at, unsigned c, int n) {
  l.g = read<FULL>(static_cast<const G*>(e.g) + at, c, n);
  if constexpr (MASTER) l.w = read<FULL>((const float*)e.master + at, c, n);
  else l.p = read<FULL>((const P*)e.p + at, c, n);
  if constexpr (BITS == 8) {
    l.mc = read_codes<FULL>((const uint8_t*)e.m + at, c, n);
    l.vc = read_codes<FULL>((const uint8_t*)e.v + at, c, n);
    l.mu = e.m_scale[at / kBlockLen];
    l.vu = e.v_scale[at / kBlockLen];
  } else {
    l.m = read<FULL>((const float*)e.m + at, c, n);
    l.v = read<FULL>((const float*)e.v + at, c, n);
  }
}

template <typename P, typename G, bool MASTER, int BITS, bool FULL>
__device__ __forceinline__ void update(const Lane<P, G, MASTER, BITS>& l, const AdamEntry& e, int64_t at, unsigned c, int n, const Factors& k,
                                       float scale, float keep, float b1, float c1, float b2, float c2, float eps) {
  float g[4], m[4], v[4], w[4], r[4];
  l.g.get(g);
  if constexpr (MASTER) l.w.get(w);
  else l.p.get(w);
  if constexpr (BITS == 8) {
    decode(l.mc, l.mu, m);
    decode(l.vc, l.vu, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= v[j];
  } else {
    l.m.get(m);
    l.v.get(v);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    g[j] *= scale;
    m[j] = fmaf(c1, g[j], b1 * m[j]);
    v[j] = fmaf(c2, g[j] * g[j], b2 * v[j]);
    r[j] = BITS == 8 ? root(v[j]) : near_root(v[j]);                // (a step off at most, like the reciprocal)
    w[j] = fmaf(w[j], keep, -k.rate * m[j] * __builtin_amdgcn_rcpf(fmaf(r[j], k.inv_root, eps)));
  }
  if constexpr (MASTER) write<FULL>(e.master + at, c, n, w);
  write<FULL>((P*)e.p + at, c, n, w);
  if constexpr (BITS == 8) {
    const float mu = unit_of(m), ru = unit_of(r), im = reciprocal(mu), ir = reciprocal(ru);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = quotient(m[j], mu, im);
      r[j] = r[j] > 0.f && r[j] < INFINITY ? fmaxf(quotient(r[j], ru, ir), kLeast) : r[j] > 0.f ? NAN : r[j];
    }
    write_codes<FULL>((uint8_t*)e.m + at, c, n, encode(m));
    write_codes<FULL>((uint8_t*)e.v + at, c, n, encode(r));
    if (c == 0) {
      e.m_scale[at / kBlockLen] = mu;
      e.v_scale[at / kBlockLen] = ru;
    }
  } else {
    write<FULL>((float*)e.m + at, c, n, m);
    write<FULL>((float*)e.v + at, c, n, v);
  }
}

template <typename P, typename G, bool MASTER, int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamArgs a) {
  constexpr int kSpan = (int)adam_span(BITS == 8), kUnroll = kSpan / kThreads / 4;
  __shared__ Factors shared;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The step's number is read by one wavefront of a workgroup.  Where it has not been counted, that one then draws a number of
  // its own; whoever draws the last one knows that all have read it, and counts the step.
  unsigned drawn = 0;
  int64_t t = 0;
  if (wave == 0) {
    t = a.step[0] + (a.counted ? 0 : 1);
    if (a.last && lane == 0) {
      unsigned one = 1;
      asm volatile("" : "+v"(one) : "v"((unsigned)t));         // (behind the read)
      drawn = __hip_atomic_fetch_add(reinterpret_cast<unsigned*>(a.step + 1), one, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
    const double first = 1.0 - power(a.beta1, (uint64_t)t), second = 1.0 - power(a.beta2, (uint64_t)t);
    if (lane == 0) shared = Factors{(float)(lr / first), (float)(1.0 / sqrt(second)), (float)lr};
  }
  __syncthreads();
  const Factors k = shared;
  const float scale = a.grad_scale ? *a.grad_scale : 1.f;
  const float b1 = (float)a.beta1, c1 = (float)(1.0 - a.beta1), b2 = (float)a.beta2, c2 = (float)(1.0 - a.beta2);
  const unsigned first = lane < a.count ? a.e[lane].first : 0xffffffffu;
  for (unsigned span = blockIdx.x; span < a.spans; span += gridDim.x) {
    const int i = __builtin_popcountll(__builtin_amdgcn_ballot_w64(first <= span)) - 1;
    const AdamEntry& e = a.e[i];
    const int64_t at0 = (int64_t)(span - e.first) * kSpan;
    // (32 bits: of a 64-bit comparison of scalars this compiler has taken the minimum by a flag that was overwritten before)
    const int left = span == e.last ? e.tail : kSpan;
    const float keep = 1.f - k.lr * e.decay;
    Lane<P, G, MASTER, BITS> l[kUnroll];
    if (left == kSpan) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) fetch<P, G, MASTER, BITS, true>(l[u], e, at0 + (u * 4 + wave) * kBlockLen, lane * 4, 0);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        update<P, G, MASTER, BITS, true>(l[u], e, at0 + (u * 4 + wave) * kBlockLen, lane * 4, 0, k, scale, keep, b1, c1, b2, c2, a.eps);
    } else {
      for (int b = wave; b * kBlockLen < left; b += 4) {
        const int64_t at = at0 + b * kBlockLen;
        const int n = left - b * kBlockLen;
        if (n >= kBlockLen) {
          fetch<P, G, MASTER, BITS, true>(l[0], e, at, lane * 4, 0);
          update<P, G, MASTER, BITS, true>(l[0], e, at, lane * 4, 0, k, scale, keep, b1, c1, b2, c2, a.eps);
        } else {
          fetch<P, G, MASTER, BITS, false>(l[0], e, at, lane * 4, n);
          update<P, G, MASTER, BITS, false>(l[0], e, at, lane * 4, n, k, scale, keep, b1, c1, b2, c2, a.eps);
        }
      }
    }
  }
  if (a.last && threadIdx.x == 0 && drawn == gridDim.x - 1) {
    a.step[0] = t;
    a.step[1] = 0;
  }
}

__global__ void adamw_count_kernel(int64_t* step) { step[0] += 1; }

template <typename P, typename G, bool MASTER> void launch(bool eight, const AdamArgs& a, unsigned grid, hipStream_t s) {
  if (eight) hipLaunchKernelGGL((adamw_kernel<P, G, MASTER, 8>), dim3(grid), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((adamw_kernel<P, G, MASTER, 32>), dim3(grid), dim3(kThreads), 0, s, a);
}

}  // namespace

int launch_adamw_count(int64_t* step, hipStream_t s) {
  hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(1), 0, s, step);
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

int launch_adamw(int kind, const AdamArgs& a, hipStream_t s) {
  constexpr unsigned kMost = 1u << 22;           // (a launch holds fewer than 2^32 threads in a dimension)
  const unsigned grid = a.spans < 1 ? 1 : a.spans < kMost ? a.spans : kMost;
  const bool eight = kind & kAdam8;
  switch (kind & ~kAdam8) {
    case 0: launch<float, float, false>(eight, a, grid, s); break;
    case kAdamGradBf16: launch<float, __bf16, false>(eight, a, grid, s); break;
    case kAdamParamBf16: launch<__bf16, float, false>(eight, a, grid, s); break;
    case kAdamParamBf16 | kAdamGradBf16: launch<__bf16, __bf16, false>(eight, a, grid, s); break;
    case kAdamParamBf16 | kAdamMaster: launch<__bf16, float, true>(eight, a, grid, s); break;
    default: launch<__bf16, __bf16, true>(eight, a, grid, s); break;
  }
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

}  // namespace seco
