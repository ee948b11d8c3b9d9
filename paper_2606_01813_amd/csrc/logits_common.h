// Device code shared by the kernels on logits: element types, vectors of 16 bytes at any element's address, sums.
#pragma once

#include <hip/hip_runtime.h>

#include "logits_args.h"

namespace caddtree {
namespace lg {

constexpr int kWave = 64;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The element types: an element of a 32-bit word to fp32, and fp32 rounded into one (to the nearest, ties to even).
struct BF16 {
  using T = __bf16;
  typedef __bf16 T2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float get(uint32_t w, int j) { return __uint_as_float(j ? w & 0xffff0000u : w << 16); }
};
struct F16 {
  using T = _Float16;
  typedef _Float16 T2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float get(uint32_t w, int j) { return (float)__builtin_bit_cast(T2, w)[j]; }
};
struct F32 {
  using T = float;
  static __device__ __forceinline__ float get(uint32_t w, int) { return __uint_as_float(w); }
};
template <typename E>
constexpr int kN = 16 / (int)sizeof(typename E::T);      // elements of 16 bytes
template <typename E>
constexpr int kEach = 4 / (int)sizeof(typename E::T);    // ... of a word

// 16 bytes of elements.  Rows start at any element (a vocabulary or a stride of any length), so a vector is
// aligned to its elements alone; the hardware takes 16-byte loads and stores at such addresses.
template <typename E>
struct Vec {
  using T = typename E::T;
  struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    u32x4 w;
  };
  u32x4 w;
  static __device__ __forceinline__ Vec load(const T* p) { return Vec{reinterpret_cast<const Loose*>(p)->w}; }
  __device__ __forceinline__ void store(T* p) const { reinterpret_cast<Loose*>(p)->w = w; }
  // vector v of a row (of fewer than 2^32 bytes; a row's start stays in scalar registers)
  static __device__ __forceinline__ Vec load(const T* row, uint32_t v) {
    return load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + v * 16u));
  }
  static __device__ __forceinline__ Vec load_at(const T* row, uint32_t byte) {
    return load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + byte));
  }
  // ... at a byte of the row, with the hint that nothing else reads it soon
  static __device__ __forceinline__ Vec load_once(const T* row, uint32_t byte) {
    return Vec{__builtin_nontemporal_load(&reinterpret_cast<const Loose*>(reinterpret_cast<const char*>(row) + byte)->w)};
  }
  __device__ __forceinline__ void stream_at(T* row, uint32_t byte) const {
    __builtin_nontemporal_store(w, &reinterpret_cast<Loose*>(reinterpret_cast<char*>(row) + byte)->w);
  }
  __device__ __forceinline__ void get(float (&x)[kN<E>]) const {
#pragma unroll
    for (int j = 0; j < kN<E>; ++j) x[j] = E::get(w[j / kEach<E>], j % kEach<E>);
  }
  __device__ __forceinline__ void set(const float (&x)[kN<E>]) {
    if constexpr (kEach<E> == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        typename E::T2 v;
        v[0] = (T)x[2 * j];
        v[1] = (T)x[2 * j + 1];
        w[j] = __builtin_bit_cast(uint32_t, v);
      }
    }
  }
  // element j of those as they are
  __device__ __forceinline__ T raw(int j) const {
    const uint32_t word = w[j / kEach<E>];                // (a copy: bit_cast of a vector's element takes the first)
    if constexpr (kEach<E> == 1) return __uint_as_float(word);
    else return __builtin_bit_cast(typename E::T2, word)[j % 2];
  }
  // Makes the registers opaque: what was unpacked of them before is not kept for use after.
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
};

template <typename E>
__device__ __forceinline__ typename E::T* row_of(const Rows& r, int64_t b, int64_t t) {
  return reinterpret_cast<typename E::T*>(r.data) + b * r.b + t * r.t;
}

// Vector v of a row that has n >= 1, or the last where there are fewer: no load waits behind a branch, and a lane past the
// row's end leaves out what it gets.  kOnce: it is not read again.
template <typename E, bool kOnce = false>
__device__ __forceinline__ Vec<E> row_vector(const typename E::T* l, int v, int n) {
  const uint32_t at = (uint32_t)min(v, n - 1);
  return kOnce ? Vec<E>::load_once(l, at * 16u) : Vec<E>::load(l, at);
}

// over the lanes of a wavefront, the result in all of them (fixed order)
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

}  // namespace lg
}  // namespace caddtree
