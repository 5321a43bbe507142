// Layer norm.  Forward: s = x + r (rounded to the rows' type where there is a residual r), mean and variance of a row of s,
// y = (s - mean) rstd gain + bias.  Backward, with n = (x - mean) rstd and e = dy gain:
//   d_x = d_in + rstd (e - mean(e) - n mean(e n)),   d_gain = sum over rows of dy n,   d_bias = sum over rows of dy.
//
// Bound by memory: every row is read once and held in registers from the first sum to the result; all of a row's loads are
// issued before the first is used.  A group of G lanes takes a row: 16 lanes for the shortest (four rows to a wavefront), a
// wavefront (no barrier then), a workgroup beyond (forward_shape, backward_shape).
// Sums are fp32 in a fixed order.  The variance is taken about the mean (a second pass over registers): with
// m0 the rounded mean, delta = mean(s - m0) corrects it, so that rows with a mean far from zero keep their precision.
#include <type_traits>

#include "row_tiles.h"
#include "train_ops.h"

namespace seco {
namespace {

constexpr int kBlock = 512;                    // threads of a workgroup that takes a row
constexpr int64_t kGridX = 1 << 22;            // workgroups along x: a launch holds fewer than 2^32 threads in a dimension

// Where a group's lane finds its k-th word of a row of d elements: at `at`, with the elements from `skip` on its own.  The
// last word of a row whose length is no multiple of V overlaps the one in front of it (both lanes then store the
// same values there); behind the end there are none (skip = V).
template <int V, int G> struct Place {
  unsigned at;
  int skip;
  __device__ __forceinline__ Place(int k, int lane, int d) {
    const int c = (k * G + lane) * V;
    at = (unsigned)(c + V <= d ? c : d - V);
    skip = c < d ? c - (int)at : V;
  }
};
// The row's number where all lanes of a wavefront share it: its address is then a scalar
template <int G> __device__ __forceinline__ int64_t row_of(int64_t row) {
  if constexpr (G < 64) return row;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)row), hi = __builtin_amdgcn_readfirstlane((unsigned)(row >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

template <typename T, int V> __device__ __forceinline__ void load_gain(const void* p, bool f32, unsigned at, float* g) {
  if (sizeof(T) == 4 || f32)
    Pack<float, V>::at(static_cast<const float*>(p), at).get(g);
  else
    Pack<T, V>::at(static_cast<const T*>(p), at).get(g);
}

// Where a lane finds its KB words, and the gain there in fp32 (ones without one)
template <typename T, int V, int G, int KB> struct Words {
  int lane, d;
  __device__ __forceinline__ Words(int lane, int d) : lane(lane), d(d) {}
  __device__ __forceinline__ Place<V, G> operator[](int k) const { return Place<V, G>(k, lane, d); }
};
template <typename T, int V, int G, int KB>
__device__ __forceinline__ void gains(const NormArgs& a, const Words<T, V, G, KB>& at, float (&gain)[KB][V]) {
#pragma unroll
  for (int k = 0; k < KB; ++k) {
#pragma unroll
    for (int j = 0; j < V; ++j) gain[k][j] = 1.f;
    if (a.gain) load_gain<T, V>(a.gain, a.gain_f32, at[k].at, gain[k]);
  }
}

// Sums over a workgroup of TH threads of N <= 16 values at a time, as scalars; sh: this call's own scratch until the call
// after the next.  Behind the barrier lane i + 16 w of every wavefront takes the share of wavefront w (and of w + 4) of value
// i, then the four lanes of a value add theirs.
template <int TH, int N> __device__ __forceinline__ void block_sums(float (&x)[N], float (*sh)[N]) {
  static_assert(N <= 16 && (N & (N - 1)) == 0 && (TH == 256 || TH == 512), "");
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lanes_sum<64>(x[i]);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) sh[wave][i] = x[i];
  __syncthreads();
  float v = sh[lane >> 4][lane & (N - 1)];
  if constexpr (TH == 512) v += sh[(lane >> 4) + 4][lane & (N - 1)];
  v = sum_across_32(sum_across_16(v));
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i));
}

// Words of the rows.  FAR: of tensors that no cache holds until they are used again (see far_apart): past the caches.
template <bool FAR, typename T, int V> __device__ __forceinline__ Pack<T, V> word_at(const T* row, unsigned c) {
  if constexpr (FAR) return Pack<T, V>::once(row, c);
  else return Pack<T, V>::at(row, c);
}
template <bool FAR, typename T, int V> __device__ __forceinline__ void word_to(const Pack<T, V>& w, T* row, unsigned c) {
  if constexpr (FAR) w.away(row, c);
  else w.to(row, c);
}

// Statistics of a row.  One that holds a NaN or an infinity has an rstd of NaN, as the formula gives it (a maximum with zero would
// take the zero), and a mean of its sum, whose deviations are NaN.
__device__ __forceinline__ float rstd_of(float var, float eps) { return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps); }
__device__ __forceinline__ float mean_of(float m0, float delta) { return fabsf(m0) < INFINITY ? m0 + delta : m0; }

// ---- forward: G lanes to a row, KB words of V elements to a lane
template <typename T, int V, int G, int KB, bool FAR>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_fwd_kernel(NormArgs a) {
  constexpr int kRows = G >= 256 ? 1 : 256 / G;
  __shared__ float sh[2][G / 64 + 1][2];
  const int lane = threadIdx.x % G;
  const int64_t row = row_of<G>(((int64_t)blockIdx.y * kGridX + blockIdx.x) * kRows + threadIdx.x / G);
  if (row >= a.rows) return;                      // (a workgroup to a row: all of it)
  const int d = (int)a.d;
  const T* x = static_cast<const T*>(a.x) + row * a.xs;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * a.rs : nullptr;
  bool bad = false;
  if (a.token) {
    int64_t t = a.token[row];
    t += t < 0 ? a.table : 0;
    bad = t < 0 || t >= a.table;
    if (bad && a.outside && lane == 0) *a.outside = 1.f;
    x = static_cast<const T*>(a.x) + (bad ? 0 : t) * a.xs;
  }
  Pack<T, V> w[KB], rw[KB];
#pragma unroll
  for (int k = 0; k < KB; ++k) w[k] = word_at<FAR, T, V>(x, Place<V, G>(k, lane, d).at);
  if (r)
#pragma unroll
    for (int k = 0; k < KB; ++k) rw[k] = word_at<FAR, T, V>(r, Place<V, G>(k, lane, d).at);
  float f[KB][V], sum[1] = {0.f};
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const Place<V, G> p(k, lane, d);
    w[k].get(f[k]);
    if (r) {
      float g[V];
      rw[k].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) f[k][j] += g[j];
      w[k] = Pack<T, V>::of(f[k]);
      w[k].get(f[k]);
    }
    if (a.token && bad) {
#pragma unroll
      for (int j = 0; j < V; ++j) f[k][j] = NAN;
      w[k] = Pack<T, V>::of(f[k]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0] += j >= p.skip ? f[k][j] : 0.f;
  }
  if constexpr (G <= 64) sum[0] = lanes_sum<G>(sum[0]);
  else block_sums<G, 1>(sum, reinterpret_cast<float(*)[1]>(sh[0]));
  const float inv = 1.f / (float)d, m0 = sum[0] * inv;
  float two[2] = {0.f, 0.f};                      // of the deviations from m0, and of their squares
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const Place<V, G> p(k, lane, d);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      f[k][j] -= m0;
      const float dev = j >= p.skip ? f[k][j] : 0.f;
      two[0] += dev;
      two[1] += dev * dev;
    }
  }
  if constexpr (G <= 64) {
    two[0] = lanes_sum<G>(two[0]);
    two[1] = lanes_sum<G>(two[1]);
  } else {
    block_sums<G, 2>(two, sh[1]);
  }
  const float delta = two[0] * inv, rstd = rstd_of(two[1] * inv - delta * delta, a.eps);
  if (lane == 0) {
    a.mean[row] = mean_of(m0, delta);
    a.rstd[row] = rstd;
  }
  T* y = static_cast<T*>(a.y) + row * a.ys;
  T* out = a.out ? static_cast<T*>(a.out) + row * a.os : nullptr;
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const Place<V, G> p(k, lane, d);
    if (p.skip >= V) continue;
    float g[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = (f[k][j] - delta) * rstd;
    if (a.gain) {
      load_gain<T, V>(a.gain, a.gain_f32, p.at, b);
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] *= b[j];
    }
    if (a.bias) {
      load_gain<T, V>(a.bias, a.gain_f32, p.at, b);
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] += b[j];
    }
    if (out) word_to<FAR>(w[k], out, p.at);
    word_to<FAR>(Pack<T, V>::of(g), y, p.at);
  }
}

// Rows longer than a workgroup's registers are walked over by words of V elements, U at a time: f(V, places, whether they are
// there); what is left behind the last whole word, by single elements.  A place is always the same thread's, so that a result
// may lie over what it is made of.
template <int V, int U, typename F> __device__ __forceinline__ void walk(int64_t d, F f) {
  const unsigned words = (unsigned)(d / V);
  for (unsigned w = threadIdx.x; w < words; w += U * kBlock) {
    unsigned at[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      there[u] = w + u * kBlock < words;
      at[u] = (there[u] ? w + u * kBlock : w) * V;
    }
    f(std::integral_constant<int, V>{}, at, there);
  }
  unsigned at[1] = {words * V + threadIdx.x};
  bool there[1] = {true};
  if (at[0] < d) f(std::integral_constant<int, 1>{}, at, there);
}

// Three walks over the row (the second and third from the caches): 4096 x 16384 fp32 with a residual 238 us, by single elements 370.
template <typename T>
__global__ __launch_bounds__(kBlock) void norm_fwd_long_kernel(NormArgs a) {
  __shared__ float sh[2][kBlock / 64][2];
  constexpr int kV = 16 / sizeof(T), kU = 4;
  const int64_t row = (int64_t)blockIdx.y * kGridX + blockIdx.x, d = a.d;
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.xs;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * a.rs : nullptr;
  bool bad = false;
  if (a.token) {
    int64_t t = a.token[row];
    t += t < 0 ? a.table : 0;
    bad = t < 0 || t >= a.table;
    if (bad && a.outside && threadIdx.x == 0) *a.outside = 1.f;
    x = static_cast<const T*>(a.x) + (bad ? 0 : t) * a.xs;
  }
  T* out = a.out ? static_cast<T*>(a.out) + row * a.os : nullptr;
  const T* s = out ? out : x;                    // the row that is normalised, from the second walk on
  float sum[1] = {0.f};
  walk<kV, kU>(d, [&](auto v, auto& at, auto& there) {
    constexpr int V = decltype(v)::value, U = std::extent<std::remove_reference_t<decltype(at)>>::value;
    Pack<T, V> w[U], rw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = Pack<T, V>::at(x, at[u]);
      if (r) rw[u] = Pack<T, V>::at(r, at[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[V], g[V];
      w[u].get(f);
      if (r) rw[u].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = bad ? NAN : r ? f[j] + g[j] : f[j];
      const Pack<T, V> rounded = Pack<T, V>::of(f);
      rounded.get(f);
      if (out && there[u]) rounded.to(out, at[u]);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += there[u] ? f[j] : 0.f;
    }
  });
  block_sums<kBlock, 1>(sum, reinterpret_cast<float(*)[1]>(sh[0]));
  const float inv = 1.f / (float)d, m0 = sum[0] * inv;
  float two[2] = {0.f, 0.f};
  walk<kV, kU>(d, [&](auto v, auto& at, auto& there) {
    constexpr int V = decltype(v)::value, U = std::extent<std::remove_reference_t<decltype(at)>>::value;
    Pack<T, V> w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = Pack<T, V>::at(s, at[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[V];
      w[u].get(f);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float dev = there[u] ? f[j] - m0 : 0.f;
        two[0] += dev;
        two[1] += dev * dev;
      }
    }
  });
  block_sums<kBlock, 2>(two, sh[1]);
  const float delta = two[0] * inv, rstd = rstd_of(two[1] * inv - delta * delta, a.eps);
  if (threadIdx.x == 0) {
    a.mean[row] = mean_of(m0, delta);
    a.rstd[row] = rstd;
  }
  T* y = static_cast<T*>(a.y) + row * a.ys;
  walk<kV, kU>(d, [&](auto v, auto& at, auto& there) {
    constexpr int V = decltype(v)::value, U = std::extent<std::remove_reference_t<decltype(at)>>::value;
    Pack<T, V> w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = Pack<T, V>::at(s, at[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[V], g[V];
      w[u].get(f);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = ((f[j] - m0) - delta) * rstd;
      if (a.gain) {
        load_gain<T, V>(a.gain, a.gain_f32, at[u], g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] *= g[j];
      }
      if (a.bias) {
        load_gain<T, V>(a.bias, a.gain_f32, at[u], g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += g[j];
      }
      if (there[u]) Pack<T, V>::of(f).to(y, at[u]);
    }
  });
}

// ---- backward.  A workgroup keeps the gain and the sums of its lanes' columns in registers and takes rows in turn, the next
// ones requested before the present ones are worked on: with one workgroup to a CU nothing else covers the arithmetic.
// What a group of lanes holds of R rows: words of x, dy and d_in, and the rows' statistics
template <typename T, int V, int KB, int R, bool IN, bool FAR> struct Held {
  Pack<T, V> x[R][KB], y[R][KB], in[IN ? R : 1][IN ? KB : 1];
  float mean[R], rstd[R];
  // d_x may be d_in, and the last word of a row may overlap one of another wavefront's: d_in is there before that one's result
  // is written, that is before the barrier of the sums
  __device__ __forceinline__ void arrived() {
    if constexpr (IN)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < KB; ++k) in[i][k].arrived();
  }
  // rows r0 .. r0 + there - 1; of the others the last one again
  template <typename At> __device__ __forceinline__ void load(const NormArgs& a, int64_t r0, int there, const At& at) {
    int64_t xs = a.xs, ys = a.ys, rs = a.rs;
    asm volatile("" : "+s"(xs), "+s"(ys), "+s"(rs));             // (or every row's address is kept through the loop)
    const T* x0 = static_cast<const T*>(a.x) + r0 * xs;
    const T* y0 = static_cast<const T*>(a.dy) + r0 * ys;
    const T* in0 = static_cast<const T*>(a.r) + r0 * rs;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = min(i, there - 1);
      mean[i] = a.mean[r0 + r];
      rstd[i] = a.rstd[r0 + r];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        x[i][k] = word_at<FAR, T, V>(x0 + r * xs, at[k].at);
        y[i][k] = word_at<FAR, T, V>(y0 + r * ys, at[k].at);
        if constexpr (IN) in[i][k] = word_at<FAR, T, V>(in0 + r * rs, at[k].at);
      }
    }
  }
};

// Columns of a lane: what it adds up
template <typename T, int V, int KB> struct Columns {
  float gain[KB][V], dg[KB][V], db[KB][V];
  Pack<T, V> own[KB];                             // masks: what is another lane's counts as a dy of zero
  template <int G> __device__ __forceinline__ Columns(const NormArgs& a, const Words<T, V, G, KB>& at) {
    gains<T, V, G, KB>(a, at, gain);
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      own[k] = Pack<T, V>::from(at[k].skip);
#pragma unroll
      for (int j = 0; j < V; ++j) dg[k][j] = db[k][j] = 0.f;
    }
  }
  // this lane's share of the sums of e and of e n over the row
  __device__ __forceinline__ void add(const Pack<T, V> (&x)[KB], const Pack<T, V> (&y)[KB], unsigned is, float mean, float rstd, float& s1,
                                      float& s2) {
    s1 = s2 = 0.f;
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      float n[V], f[V];
      x[k].get(n);
      (y[k] & own[k] & is).get(f);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        n[j] = (n[j] - mean) * rstd;
        dg[k][j] += f[j] * n[j];
        db[k][j] += f[j];
        f[j] *= gain[k][j];
        s1 += f[j];
        s2 += f[j] * n[j];
      }
    }
  }
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int k = 0; k < KB; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) here(dg[k][j]), here(db[k][j]);
  }
  // word k of d_x; s1, s2: mean(e), mean(e n)
  __device__ __forceinline__ void word(int k, const Pack<T, V>& x, const Pack<T, V>& y, float mean, float rstd, float s1, float s2,
                                       float (&f)[V]) const {
    float n[V];
    x.get(n);
    y.get(f);
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = rstd * (f[j] * gain[k][j] - s1 - (n[j] - mean) * rstd * s2);
  }
};

// G <= 64 lanes to a row: no barrier in the loop.  At the end the groups' sums meet in LDS, behind one barrier, and leave as the
// workgroup's row of the parts, in the order of the wavefronts.  The last row is taken behind the loop, so that nothing is
// requested that is not there (with both: 2048 x 1024 bf16 10.0 -> 9.0 us, its sums included).
template <typename T, int V, int G, int KB, bool IN>
__global__ __launch_bounds__(kBlock) void norm_bwd_rows_kernel(NormArgs a) {
  constexpr int kRows = kBlock / G, kWaves = kBlock / 64, kCols = G * KB * V, kOwn = (kCols + kBlock - 1) / kBlock;
  __shared__ float sh[2][kWaves][kCols];
  const int lane = threadIdx.x % G, wave = threadIdx.x >> 6, d = (int)a.d;
  const float inv = 1.f / (float)d;
  const Words<T, V, G, KB> at(lane, d);
  Columns<T, V, KB> c(a, at);
  int64_t row = row_of<G>((int64_t)blockIdx.x * kRows + threadIdx.x / G);
  const int64_t step = (int64_t)a.blocks * kRows;
  Held<T, V, KB, 1, IN, false> now, next;
  auto take_row = [&]() {
    float s1, s2;
    c.add(now.x[0], now.y[0], 0xffffffffu, now.mean[0], now.rstd[0], s1, s2);
    c.settle();
    s1 = lanes_sum<G>(s1) * inv;
    s2 = lanes_sum<G>(s2) * inv;
    T* out = static_cast<T*>(a.out) + row * a.os;
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      float f[V];
      now.x[0][k].renew(s2);
      now.y[0][k].renew(s2);
      c.word(k, now.x[0][k], now.y[0][k], now.mean[0], now.rstd[0], s1, s2, f);
      if constexpr (IN) {
        float g[V];
        now.in[0][k].get(g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += g[j];
      }
      if (at[k].skip < V) Pack<T, V>::of(f).to(out, at[k].at);
    }
  };
  if (row < a.rows) {
    now.load(a, row, 1, at);
    for (; row + step < a.rows; row += step) {
      next.load(a, row + step, 1, at);
      take_row();
      now = next;
    }
    take_row();
  }
  if (!a.parts) return;
  float old[2][kOwn];                             // of this thread's columns, under the sums over the wavefronts
  float* part[2] = {a.parts + (int64_t)blockIdx.x * d, a.parts + ((int64_t)a.part_rows + blockIdx.x) * d};
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int i = k * kBlock + threadIdx.x;
      old[q][k] = a.accumulate ? part[q][min(i, d - 1)] : 0.f;
    }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    auto& s = q ? c.db : c.dg;
    if constexpr (G == 16)
#pragma unroll
      for (int k = 0; k < KB; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) s[k][j] = sum_across_32(sum_across_16(s[k][j]));
    if ((threadIdx.x & 63) < G)
#pragma unroll
      for (int k = 0; k < KB; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j >= at[k].skip) sh[q][wave][at[k].at + j] = s[k][j];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int i = k * kBlock + threadIdx.x;
      if (i >= d) break;
      float f = sh[q][0][i];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) f += sh[q][w][i];
      part[q][i] = old[q][k] + f;
    }
}

// A workgroup to a row, R rows at a time: one barrier for their 2 R sums.  AHEAD: the next rows are requested under the present
// ones; four words of bf16 to a lane leave no registers for that.
template <typename T, int V, int KB, int R, bool AHEAD, bool IN, bool FAR>
__global__ __launch_bounds__(kBlock) void norm_bwd_block_kernel(NormArgs a) {
  __shared__ float sh[2][kBlock / 64][2 * R];
  const int d = (int)a.d;
  const float inv = 1.f / (float)d;
  const Words<T, V, kBlock, KB> at(threadIdx.x, d);
  Columns<T, V, KB> c(a, at);
  int64_t r0 = (int64_t)blockIdx.x * R;
  const int64_t step = (int64_t)a.blocks * R;
  auto rows_at = [&](int64_t r) { return (int)min((int64_t)R, a.rows - r); };
  Held<T, V, KB, R, IN, FAR> now, next;
  if (AHEAD && r0 < a.rows) now.load(a, r0, rows_at(r0), at);
  int turn = 0;
  for (; r0 < a.rows; r0 += step, turn ^= 1) {
    const int there = rows_at(r0);
    if constexpr (AHEAD) {
      const int64_t r1 = r0 + step < a.rows ? r0 + step : r0;
      next.load(a, r1, rows_at(r1), at);
    } else {
      now.load(a, r0, there, at);
    }
    float s[2 * R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (i > 0)                                  // one row's fp32 values at a time
#pragma unroll
        for (int k = 0; k < KB; ++k) now.x[i][k].renew(s[2 * i - 1]), now.y[i][k].renew(s[2 * i - 1]);
      c.add(now.x[i], now.y[i], i < there ? 0xffffffffu : 0u, now.mean[i], now.rstd[i], s[2 * i], s[2 * i + 1]);
    }
    c.settle();
    if (KB == 4 || d % V) now.arrived();          // (asked of every row 16384 x 4096 bf16 take 119 us instead of 116; asked, four words spill)
    block_sums<kBlock, 2 * R>(s, sh[turn]);
    int64_t os = a.os;
    asm volatile("" : "+s"(os));
    T* out0 = static_cast<T*>(a.out) + r0 * os;
    float last = s[0];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float s1 = s[2 * i] * inv, s2 = s[2 * i + 1] * inv;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        float f[V];
        now.x[i][k].renew(last);
        now.y[i][k].renew(last);
        c.word(k, now.x[i][k], now.y[i][k], now.mean[i], now.rstd[i], s1, s2, f);
        if constexpr (IN) {
          float g[V];
          now.in[i][k].get(g);
#pragma unroll
          for (int j = 0; j < V; ++j) f[j] += g[j];
        }
        last = f[V - 1];
        if (i < there && at[k].skip < V) word_to<FAR>(Pack<T, V>::of(f), out0 + i * os, at[k].at);
      }
    }
    if constexpr (AHEAD) now = next;
  }
  if (!a.parts) return;
  float* part = a.parts + (int64_t)blockIdx.x * d;
  float* part_b = part + (int64_t)a.part_rows * d;
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= at[k].skip) {
        float *g = part + at[k].at + j, *b = part_b + at[k].at + j;
        *g = (a.accumulate ? *g : 0.f) + c.dg[k][j];
        *b = (a.accumulate ? *b : 0.f) + c.db[k][j];
      }
}

// Rows longer than that: two walks over R rows side by side; the sums of a column are kept in the workgroup's row of the parts,
// which is read and written once for the R rows.  Single elements instead of words: 4096 x 16384 fp32 with d_in 1191 us, now 309 (floor
// 203; eight fp32 words to a lane in registers spill).  One row or four: 1000 x 16384 fp32 104 / 78; up to 512 rows there are
// too few groups of four for the CUs (600 rows 63 / 44).
template <typename T, int R>
__global__ __launch_bounds__(kBlock) void norm_bwd_long_kernel(NormArgs a) {
  __shared__ float sh[2][kBlock / 64][2 * R];
  constexpr int kV = 16 / sizeof(T), kU = R == 1 ? 4 : 1;
  const int64_t d = a.d;
  const float inv = 1.f / (float)d;
  float* part = a.parts ? a.parts + (int64_t)blockIdx.x * d : nullptr;
  float* part_b = part ? part + (int64_t)a.part_rows * d : nullptr;
  bool add = a.accumulate;
  int turn = 0;
  if (part && !add && (int64_t)blockIdx.x * R >= a.rows)         // (no rows at all)
    for (int64_t c = threadIdx.x; c < d; c += kBlock) part[c] = part_b[c] = 0.f;
  for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.rows; r0 += (int64_t)a.blocks * R, turn ^= 1, add = true) {
    const int rows = (int)min((int64_t)R, a.rows - r0);
    float mean[R], rstd[R], s[2 * R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t r = r0 + min(i, rows - 1);
      mean[i] = a.mean[r];
      rstd[i] = a.rstd[r];
      s[2 * i] = s[2 * i + 1] = 0.f;
    }
    // row i of a tensor (of those that are not there the last one), found anew: kept, R rows of four tensors spill
    auto row = [&](auto* base, int64_t stride, int i) {
      asm volatile("" : "+s"(stride));
      return base + (r0 + min(i, rows - 1)) * stride;
    };
    const T *xs = static_cast<const T*>(a.x), *dys = static_cast<const T*>(a.dy), *ins = static_cast<const T*>(a.r);
    auto gain_at = [&](auto v, unsigned at, float* g) {
      constexpr int V = decltype(v)::value;
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = 1.f;
      if (a.gain) load_gain<T, V>(a.gain, a.gain_f32, at, g);
    };
    walk<kV, kU>(d, [&](auto v, auto& at, auto& there) {
      constexpr int V = decltype(v)::value, U = std::extent<std::remove_reference_t<decltype(at)>>::value;
      Pack<T, V> xw[U][R], yw[U][R];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          xw[u][i] = Pack<T, V>::at(row(xs, a.xs, i), at[u]);
          yw[u][i] = Pack<T, V>::at(row(dys, a.ys, i), at[u]);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float g[V];
        gain_at(v, at[u], g);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          float n[V], e[V];
          xw[u][i].get(n);
          yw[u][i].get(e);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            e[j] = there[u] ? e[j] * g[j] : 0.f;
            s[2 * i] += e[j];
            s[2 * i + 1] += there[u] ? e[j] * ((n[j] - mean[i]) * rstd[i]) : 0.f;
          }
        }
      }
    });
    block_sums<kBlock, 2 * R>(s, sh[turn]);
#pragma unroll
    for (int i = 0; i < 2 * R; ++i) s[i] *= inv, here(s[i]);     // (vector registers: the scalar ones are all taken)
    walk<kV, kU>(d, [&](auto v, auto& at, auto& there) {
      constexpr int V = decltype(v)::value, U = std::extent<std::remove_reference_t<decltype(at)>>::value;
      Pack<T, V> xw[U][R], yw[U][R], iw[U][R];
      Pack<float, V> old[U], old_b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          xw[u][i] = Pack<T, V>::at(row(xs, a.xs, i), at[u]);
          yw[u][i] = Pack<T, V>::at(row(dys, a.ys, i), at[u]);
          if (a.r) iw[u][i] = Pack<T, V>::at(row(ins, a.rs, i), at[u]);
        }
        if (part && add) {
          old[u] = Pack<float, V>::at(part, at[u]);
          old_b[u] = Pack<float, V>::at(part_b, at[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float g[V], dg[V], db[V];
        gain_at(v, at[u], g);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[j] = db[j] = 0.f;
        if (part && add) {
          old[u].get(dg);
          old_b[u].get(db);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          float n[V], y[V], f[V];
          xw[u][i].get(n);
          yw[u][i].get(y);
#pragma unroll
          for (int j = 0; j < V; ++j) f[j] = 0.f;
          if (a.r) iw[u][i].get(f);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            n[j] = (n[j] - mean[i]) * rstd[i];
            dg[j] += i < rows ? y[j] * n[j] : 0.f;
            db[j] += i < rows ? y[j] : 0.f;
            f[j] += rstd[i] * (y[j] * g[j] - s[2 * i] - n[j] * s[2 * i + 1]);
          }
          if (i < rows && there[u]) Pack<T, V>::of(f).to(row(static_cast<T*>(a.out), a.os, i), at[u]);
        }
        if (part && there[u]) {
          Pack<float, V>::of(dg).to(part, at[u]);
          Pack<float, V>::of(db).to(part_b, at[u]);
        }
      }
    });
  }
}

// d_gain (blockIdx.y 0) or d_bias: 32 columns to a workgroup, 32 groups of 8 lanes, each every 32nd block's share in ascending
// order, then the groups in theirs.
template <typename T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const float* parts, int blocks, int64_t d, T* d_gain, T* d_bias) {
  __shared__ float sh[32][33];
  const float* from = parts + (int64_t)blockIdx.y * blocks * d;
  T* to = blockIdx.y ? d_bias : d_gain;
  if (!to) return;
  const int group = threadIdx.x >> 3, l8 = threadIdx.x & 7;
  const int64_t c0 = (int64_t)blockIdx.x * 32 + l8 * 4;
  float f[4] = {0.f, 0.f, 0.f, 0.f};
  if (c0 + 4 <= d) {
#pragma unroll 8
    for (int b = group; b < blocks; b += 32) {
      float x[4];
      Pack<float, 4>::at(from + b * d + c0).get(x);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] += x[j];
    }
  } else {
    for (int b = group; b < blocks; b += 32)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + j < d) f[j] += from[b * d + c0 + j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) sh[group][l8 * 4 + j] = f[j];
  __syncthreads();
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || c >= d) return;
  float s = sh[0][threadIdx.x];
#pragma unroll
  for (int g = 1; g < 32; ++g) s += sh[g][threadIdx.x];
  to[c] = (T)s;
}

// A call of few rows: one launch, without parts.  The statistics are known, so that the sums of the columns need nothing from the
// rows' workgroups (the first a.blocks): the ones behind them walk down the rows, 4 words of columns to a workgroup, 128
// groups of lanes that take every 128th row each, four at a time, then a tree over the groups.  Two workgroups read a cache line
// of 128 bytes: `which` puts them on one XCD (1024 x 8192 bf16 22.7 -> 18.4 us).
template <typename T, int V> __device__ __forceinline__ void column_sums(const NormArgs& a, int which) {
  __shared__ float sh[kBlock / 64][4][2][V];
  constexpr int kGroups = kBlock / 4, kAhead = 4;
  const int lane = threadIdx.x & 3, rows = (int)a.rows;
  const Place<V, 4> at(which, lane, (int)a.d);
  float s[2][V];
#pragma unroll
  for (int j = 0; j < V; ++j) s[0][j] = s[1][j] = 0.f;
  for (int r0 = threadIdx.x >> 2; r0 < rows; r0 += kAhead * kGroups) {
    Pack<T, V> x[kAhead], y[kAhead];
    float mean[kAhead], rstd[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t r = r0 + i * kGroups < rows ? r0 + i * kGroups : r0;
      x[i] = Pack<T, V>::at(static_cast<const T*>(a.x) + r * a.xs, at.at);
      y[i] = Pack<T, V>::at(static_cast<const T*>(a.dy) + r * a.ys, at.at);
      mean[i] = a.mean[r];
      rstd[i] = a.rstd[r];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool is = r0 + i * kGroups < rows;
      float n[V], f[V];
      x[i].get(n);
      y[i].get(f);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s[0][j] += is ? f[j] * ((n[j] - mean[i]) * rstd[i]) : 0.f;
        s[1][j] += is ? f[j] : 0.f;
      }
    }
  }
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float f = s[k][j];
      f += with_partner<0x128>(f);                // lane i - 8 of the same 16, in turn
      f += with_partner<0x124>(f);                // lane i - 4
      f = sum_across_32(sum_across_16(f));
      if ((threadIdx.x & 63) < 4) sh[wave][lane][k][j] = f;
    }
  __syncthreads();
  if (threadIdx.x >= 8 * V) return;
  const int l = threadIdx.x / (2 * V), k = threadIdx.x / V & 1, j = threadIdx.x % V;
  const Place<V, 4> to(which, l, (int)a.d);
  void* out = k ? a.d_bias : a.d_gain;
  if (j < to.skip || !out) return;
  float f = sh[0][l][k][j];
#pragma unroll
  for (int w = 1; w < kBlock / 64; ++w) f += sh[w][l][k][j];
  if (a.accumulate) static_cast<float*>(out)[to.at + j] += f;
  else if (sizeof(T) == 4 || a.gain_f32) static_cast<float*>(out)[to.at + j] = f;
  else static_cast<T*>(out)[to.at + j] = (T)f;
}
template <typename T, int V, int G, int KB, bool IN>
__global__ __launch_bounds__(kBlock) void norm_bwd_few_kernel(NormArgs a) {
  __shared__ float sh[kBlock / 64][2];
  if ((int)blockIdx.x >= a.blocks) {
    const int b = (int)blockIdx.x - a.blocks, n = (int)gridDim.x - a.blocks;
    return column_sums<T, V>(a, b < n / 16 * 16 ? b / 16 * 16 + b % 8 * 2 + b / 8 % 2 : b);
  }
  const int d = (int)a.d;
  const Words<T, V, G, KB> at(threadIdx.x % G, d);
  const int64_t row = row_of<G>((int64_t)blockIdx.x * (kBlock / G) + threadIdx.x / G);
  if (row >= a.rows) return;                      // (a workgroup to a row: never)
  Held<T, V, KB, 1, IN, false> now;
  now.load(a, row, 1, at);
  Columns<T, V, KB> c(a, at);
  float s[2];
  c.add(now.x[0], now.y[0], 0xffffffffu, now.mean[0], now.rstd[0], s[0], s[1]);
  if constexpr (G > 64) {
    now.arrived();
    block_sums<G, 2>(s, sh);
  } else {
    s[0] = lanes_sum<G>(s[0]);
    s[1] = lanes_sum<G>(s[1]);
  }
  const float inv = 1.f / (float)d;
  T* out = static_cast<T*>(a.out) + row * a.os;
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    float f[V], g[V];
    c.word(k, now.x[0][k], now.y[0][k], now.mean[0], now.rstd[0], s[0] * inv, s[1] * inv, f);
    if constexpr (IN) {
      now.in[0][k].get(g);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] += g[j];
    }
    if (at[k].skip < V) Pack<T, V>::of(f).to(out, at[k].at);
  }
}

// f is called with the elements of a word, the lanes to a row and the words to a lane.
template <int V, int G, int KB, typename F> bool take(F f) {
  f(std::integral_constant<int, V>{}, std::integral_constant<int, G>{}, std::integral_constant<int, KB>{});
  return true;
}

// Forward, by the words w of a row (16 bytes; rows shorter than that: single elements): 16 lanes up to 32, a wavefront up to 128,
// then a workgroup, so that no lane has more to load than it keeps in flight at full occupancy.  us for x + residual -> x_out, y:
//   bf16 2048 elements, a wavefront with four words / 256 lanes with one: 8 rows 4.5 / 3.0, 1024 8.2 / 7.3, 16384 53.8 / 50.7
//   128 words and few rows, a wavefront / 256 lanes: 128 rows of 1024 bf16 3.8 / 3.3, but 1024 rows 5.5 / 5.9
//   256 lanes with two words where 512 would be idle by a quarter, once there are rows for every wavefront slot: 16384 rows of 1027
//   fp32 63 / 54, of 3000 bf16 81 / 74, but 2048 fp32 92 / 99 and 8 rows of 1027 2.8 / 3.0.
template <typename T, typename F> bool forward_shape(int64_t rows, int64_t d, F f) {
  constexpr int V = 16 / sizeof(T);
  if (d < V) return take<1, 16, 1>(f);
  const int64_t w = (d + V - 1) / V;
  if (w <= 16) return take<V, 16, 1>(f);
  if (w <= 32) return take<V, 16, 2>(f);
  if (w <= 64) return take<V, 64, 1>(f);
  if (w <= 128 && rows > 512) return take<V, 64, 2>(f);
  if (w <= 256) return take<V, 256, 1>(f);
  if (w <= 384 && rows >= 2048) return take<V, 256, 2>(f);
  if (w <= 512) return take<V, kBlock, 1>(f);
  if (w <= 1024) return take<V, kBlock, 2>(f);
  if (w <= 2048) return take<V, kBlock, 4>(f);
  return false;
}
// Backward: a wavefront up to 256 words, whose sums then take half of its registers; a workgroup beyond.  FEW: no sums are kept.
template <typename T, bool FEW = false, typename F> bool backward_shape(int64_t d, F f) {
  constexpr int V = 16 / sizeof(T);
  if (d < V) return take<1, 16, 1>(f);
  const int64_t w = (d + V - 1) / V;
  if (w <= 16) return take<V, 16, 1>(f);
  if (w <= 32) return take<V, 16, 2>(f);
  if (w <= 64) return take<V, 64, 1>(f);
  if (w <= 128) return take<V, 64, 2>(f);
  if (w <= 256) return take<V, 64, 4>(f);
  if (w <= 512) return take<V, kBlock, 1>(f);
  if (w <= 1024) return take<V, kBlock, 2>(f);
  if (w <= 2048) return take<V, kBlock, 4>(f);
  if constexpr (FEW && sizeof(T) == 4)
    if (w <= 4096) return take<V, kBlock, 8>(f);
  return false;
}

// Whether a call's results are more than the 256 MiB of the last cache, so that nothing of them is there when they are read:
// its words then go past the caches.  Only for whole 16-byte words at their places: the others share lines with their
// neighbours.  us with / without: backward 16384 x 8192 bf16 150 / 164; but a second norm behind one of 8192 x 4096 93 / 84.
bool far_apart(const NormArgs& a, int elem, int results) {
  const int64_t per = 16 / elem;
  for (int64_t n : {a.d, a.xs, a.rs, a.os, a.ys})
    if (n % per) return false;
  for (const void* p : {a.x, a.r, (const void*)a.out, a.dy, (const void*)a.y})
    if (reinterpret_cast<uintptr_t>(p) & 15u) return false;
  return a.rows * a.d * elem * results >= (int64_t)1 << 28;
}
dim3 rows_grid(int64_t workgroups) {
  return dim3((unsigned)(workgroups < kGridX ? workgroups : kGridX), (unsigned)((workgroups + kGridX - 1) / kGridX));
}

template <typename T> int norm_fwd(const NormArgs& a, hipStream_t s) {
  const bool done = forward_shape<T>(a.rows, a.d, [&](auto v, auto g, auto kb) {
    constexpr int G = decltype(g)::value, kRows = G >= 256 ? 1 : 256 / G;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, rows_grid((a.rows + kRows - 1) / kRows), dim3(G > 256 ? G : 256), 0, s, a); };
    if constexpr (G >= 256)
      if (far_apart(a, sizeof(T), a.out ? 2 : 1)) return launch(norm_fwd_kernel<T, decltype(v)::value, G, decltype(kb)::value, true>);
    launch(norm_fwd_kernel<T, decltype(v)::value, G, decltype(kb)::value, false>);
  });
  if (!done) hipLaunchKernelGGL(norm_fwd_long_kernel<T>, rows_grid(a.rows), dim3(kBlock), 0, s, a);
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

template <typename T> constexpr bool ahead(int kb) { return kb < 4 || sizeof(T) == 4; }
template <typename T> constexpr int rows_at_once(int kb) { return ahead<T>(kb) ? 4 / kb : 2; }
int rows_of_long(int64_t rows) { return rows <= 2 * SECO_NORM_BLOCKS ? 1 : 4; }   // (see norm_bwd_long_kernel)
template <typename T> int rows_of_block(int64_t rows, int64_t d) {      // rows that a workgroup of the backward takes at a time
  int n = rows_of_long(rows);
  backward_shape<T>(d, [&](auto, auto g, auto kb) {
    constexpr int G = decltype(g)::value;
    n = G <= 64 ? kBlock / G : rows_at_once<T>(decltype(kb)::value);
  });
  return n;
}

template <typename T> int norm_bwd(const NormArgs& a, hipStream_t s) {
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.blocks), dim3(kBlock), 0, s, a); };
  const bool done = backward_shape<T>(a.d, [&](auto v, auto g, auto kb) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value, KB = decltype(kb)::value;
    if constexpr (G <= 64) a.r ? launch(norm_bwd_rows_kernel<T, V, G, KB, true>) : launch(norm_bwd_rows_kernel<T, V, G, KB, false>);
    else {
      constexpr int R = rows_at_once<T>(KB);
      constexpr bool kAhead = ahead<T>(KB);
      if (far_apart(a, sizeof(T), 1)) a.r ? launch(norm_bwd_block_kernel<T, V, KB, R, kAhead, true, true>) : launch(norm_bwd_block_kernel<T, V, KB, R, kAhead, false, true>);
      else a.r ? launch(norm_bwd_block_kernel<T, V, KB, R, kAhead, true, false>) : launch(norm_bwd_block_kernel<T, V, KB, R, kAhead, false, false>);
    }
  });
  if (!done) rows_of_long(a.rows) == 1 ? launch(norm_bwd_long_kernel<T, 1>) : launch(norm_bwd_long_kernel<T, 4>);
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

template <typename T> int norm_bwd_few(NormArgs a, bool rows, bool sums, hipStream_t s) {
  backward_shape<T, true>(a.d, [&](auto v, auto g, auto kb) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value, KB = decltype(kb)::value, kRows = kBlock / G;
    a.blocks = rows ? (int)((a.rows + kRows - 1) / kRows) : 0;
    const unsigned grid = (unsigned)(a.blocks + (sums ? (a.d + 4 * V - 1) / (4 * V) : 0));
    if (a.r) hipLaunchKernelGGL((norm_bwd_few_kernel<T, V, G, KB, true>), dim3(grid), dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL((norm_bwd_few_kernel<T, V, G, KB, false>), dim3(grid), dim3(kBlock), 0, s, a);
  });
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

}  // namespace

// Up to 1280 rows; beyond, the walk down the rows is the longest way.  us, one launch / parts and their sums, tensors out of memory:
// bf16 1100 x 100 6.2 / 8.3, 1100 x 1024 9.2 / 9.6, 1100 x 4096 14.5 / 21.1, 1000 x 16384 47 / 60, fp32 300 x 15520 24 / 34, 1000 x 8192
// 34.6 / 39.3; 1500 rows between 6.6 / 7.8 (100 elements) and 11.4 / 10.6 (1000), 2048 x 1024 14.3 / 10.2, 3000 x 512 18.2 / 7.8.
bool norm_few(int64_t rows, int64_t d) { return rows >= 1 && rows <= kNormFewRows && d <= kNormFewLength; }
int launch_norm_bwd_few(const NormArgs& a, bool rows, bool sums, hipStream_t s) {
  return a.dtype == SECO_BF16 ? norm_bwd_few<__bf16>(a, rows, sums, s) : norm_bwd_few<float>(a, rows, sums, s);
}

int norm_blocks(int64_t rows, int64_t d, int dtype) {
  const int per = dtype == SECO_BF16 ? rows_of_block<__bf16>(rows, d) : rows_of_block<float>(rows, d);
  const int64_t n = (rows + per - 1) / per;
  return (int)(n < 1 ? 1 : n < SECO_NORM_BLOCKS ? n : SECO_NORM_BLOCKS);
}

int launch_norm_fwd(const NormArgs& a, hipStream_t s) { return a.dtype == SECO_BF16 ? norm_fwd<__bf16>(a, s) : norm_fwd<float>(a, s); }
int launch_norm_bwd(const NormArgs& a, hipStream_t s) { return a.dtype == SECO_BF16 ? norm_bwd<__bf16>(a, s) : norm_bwd<float>(a, s); }

int launch_norm_sums(const float* parts, int blocks, int64_t d, void* d_gain, void* d_bias, int gain_f32, hipStream_t s) {
  const dim3 grid((unsigned)((d + 31) / 32), 2);
  if (gain_f32)
    hipLaunchKernelGGL(norm_sums_kernel<float>, grid, dim3(256), 0, s, parts, blocks, d, (float*)d_gain, (float*)d_bias);
  else
    hipLaunchKernelGGL(norm_sums_kernel<__bf16>, grid, dim3(256), 0, s, parts, blocks, d, (__bf16*)d_gain, (__bf16*)d_bias);
  return hipGetLastError() == hipSuccess ? SECO_OK : SECO_ERR_LAUNCH;
}

}  // namespace seco
