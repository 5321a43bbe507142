// What the kernels over rows and flat tensors share: words of a few elements, and sums over the lanes that share a row.
#pragma once
#include <hip/hip_runtime.h>

namespace seco {
namespace {

// V consecutive elements, moved by one access.  Only the elements' own alignment is asked for: gfx950 loads and stores 16
// bytes from any element on, so that rows of odd lengths and views that start anywhere take the same path as aligned ones.
// (Held as 32-bit words: as an array of bf16 every element would take a register of its own.)
template <typename T, int V> struct Pack {
  static constexpr int kWords = (int)(sizeof(T) * V + 3) / 4;
  unsigned w[kWords];
  __device__ __forceinline__ static Pack at(const T* p) {
    Pack x;
    if constexpr (sizeof(T) * V >= 4) {
      typedef unsigned words __attribute__((ext_vector_type(kWords)));
      words u;
      __builtin_memcpy(&u, p, sizeof(T) * V);
#pragma unroll
      for (int i = 0; i < kWords; ++i) x.w[i] = u[i];
    } else {
      x.w[0] = *reinterpret_cast<const unsigned short*>(p);
    }
    return x;
  }
  // the same for what is not used again: marked so that it does not push other data out of the caches
  __device__ __forceinline__ static Pack once(const T* p) {
    if constexpr (sizeof(T) * V >= 4) {
      typedef unsigned words __attribute__((ext_vector_type(kWords)));
      typedef words loose __attribute__((aligned(sizeof(T))));
      const words u = __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
      Pack x;
#pragma unroll
      for (int i = 0; i < kWords; ++i) x.w[i] = u[i];
      return x;
    } else {
      return at(p);
    }
  }
  __device__ __forceinline__ void away(T* p) const {
    if constexpr (sizeof(T) * V >= 4) {
      typedef unsigned words __attribute__((ext_vector_type(kWords)));
      typedef words loose __attribute__((aligned(sizeof(T))));
      words u;
#pragma unroll
      for (int i = 0; i < kWords; ++i) u[i] = w[i];
      __builtin_nontemporal_store(u, reinterpret_cast<loose*>(p));
    } else {
      to(p);
    }
  }
  __device__ __forceinline__ static Pack once(const T* row, unsigned c) {
    return once(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + c * (unsigned)sizeof(T)));
  }
  __device__ __forceinline__ void away(T* row, unsigned c) const {
    away(reinterpret_cast<T*>(reinterpret_cast<char*>(row) + c * (unsigned)sizeof(T)));
  }
  // element c of a row (rows are shorter than 2^32 bytes: a scalar base and a 32-bit offset)
  __device__ __forceinline__ static Pack at(const T* row, unsigned c) {
    return at(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + c * (unsigned)sizeof(T)));
  }
  __device__ __forceinline__ void to(T* row, unsigned c) const {
    to(reinterpret_cast<T*>(reinterpret_cast<char*>(row) + c * (unsigned)sizeof(T)));
  }
  __device__ __forceinline__ void to(T* p) const {
    if constexpr (sizeof(T) * V >= 4) {
      typedef unsigned words __attribute__((ext_vector_type(kWords)));
      words u;
#pragma unroll
      for (int i = 0; i < kWords; ++i) u[i] = w[i];
      __builtin_memcpy(p, &u, sizeof(T) * V);
    } else {
      *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int j = 0; j < V; ++j)
      f[j] = __builtin_bit_cast(float, sizeof(T) == 4 ? w[j] : j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
  __device__ __forceinline__ static Pack of(const float* f) {
    Pack x;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < V; ++j) x.w[j] = __builtin_bit_cast(unsigned, f[j]);
    } else if constexpr (V == 1) {
      x.w[0] = __builtin_bit_cast(unsigned short, (__bf16)f[0]);
    } else {
      typedef __bf16 two __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int j = 0; j < V; j += 2) x.w[j / 2] = __builtin_bit_cast(unsigned, two{(__bf16)f[j], (__bf16)f[j + 1]});
    }
    return x;
  }
  // all ones where j >= first (elements), zero elsewhere; and the elements that a mask leaves
  __device__ __forceinline__ static Pack from(int first) {
    Pack m;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) m.w[i] = i >= first ? 0xffffffffu : 0u;
      else m.w[i] = (2 * i >= first ? 0xffffu : 0u) | (2 * i + 1 >= first ? 0xffff0000u : 0u);
      asm volatile("" : "+v"(m.w[i]));           // (kept as a word: as a comparison's result it would take two scalars)
    }
    return m;
  }
  __device__ __forceinline__ Pack operator&(const Pack& m) const {
    Pack x;
#pragma unroll
    for (int i = 0; i < kWords; ++i) x.w[i] = w[i] & m.w[i];
    return x;
  }
  __device__ __forceinline__ Pack operator&(unsigned m) const {
    Pack x;
#pragma unroll
    for (int i = 0; i < kWords; ++i) x.w[i] = w[i] & m;
    return x;
  }
  // The load of this word has returned here
  __device__ __forceinline__ void arrived() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
  }
  // What is computed from the elements behind this point waits for `after`, and is not what was computed from them in front of
  // it: the compiler would keep the fp32 values of several rows in registers instead of their half as large words.
  __device__ __forceinline__ void renew(float after) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) asm("" : "+v"(w[i]) : "v"(after));
  }
};

// The value is computed here: left to itself the compiler moves sums to the end of a loop's body and keeps what they are made
// of in registers until then.
__device__ __forceinline__ void here(float& x) { asm volatile("" : "+v"(x)); }

// x + (x of the lane that the DPP control names).  Every lane has a partner within its row of 16.
template <int CTRL> __device__ __forceinline__ float with_partner(float x) {
  const int i = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}
// Lanes i ^ 16 and i ^ 32 (each pair of results holds a lane's value and its partner's, in the order of the lanes)
__device__ __forceinline__ float sum_across_16(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float sum_across_32(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float max_across_16(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float max_across_32(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
// Sum over groups of 16 or of all 64 lanes, in every lane and in one order: pairs, quads, halves of a row of 16, rows.  All
// lanes of a group must be active.
template <int G> __device__ __forceinline__ float lanes_sum(float x) {
  static_assert(G == 16 || G == 64, "");
  x += with_partner<0xB1>(x);      // quad_perm [1, 0, 3, 2]
  x += with_partner<0x4E>(x);      // quad_perm [2, 3, 0, 1]
  x += with_partner<0x141>(x);     // lane 7 - i of the same 8
  x += with_partner<0x140>(x);     // lane 15 - i of the same 16
  if constexpr (G == 64) x = sum_across_32(sum_across_16(x));
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, with_partner<0xB1>(x));
  x = fmaxf(x, with_partner<0x4E>(x));
  x = fmaxf(x, with_partner<0x141>(x));
  x = fmaxf(x, with_partner<0x140>(x));
  return max_across_32(max_across_16(x));
}

}  // namespace
}  // namespace seco
