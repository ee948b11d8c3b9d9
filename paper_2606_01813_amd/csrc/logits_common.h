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

// Sequences are numbered in a grid's second and third dimension, which hold 65535 each; the last workgroups may have none.
inline dim3 grid_of(int64_t x, int32_t B) {
  const unsigned y = B < 32768 ? (unsigned)B : 32768u;
  return dim3((unsigned)x, y, ((unsigned)B + y - 1) / y);
}
__device__ __forceinline__ int sequence() { return (int)(blockIdx.z * gridDim.y + blockIdx.y); }

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

// Over the lanes of a wavefront, the result in all of them, in a fixed order: pairs, fours, eights (a mirrored eight holds
// the other four's), sixteens, then rows of 16 and halves swapped between two registers.  No trip through LDS: with
// shuffles, which go through it, 64 rows' loss and gradient took 21.2 us instead of 19.5, one row's 13.4 instead of 11.7.
template <int kControl>
__device__ __forceinline__ uint32_t moved(uint32_t w) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, kControl, 0xf, 0xf, true);
}
template <int kControl>
__device__ __forceinline__ float moved(float v) { return __uint_as_float(moved<kControl>(__float_as_uint(v))); }
template <int kControl>
__device__ __forceinline__ double moved(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)moved<kControl>((uint32_t)(w >> 32)) << 32 | moved<kControl>((uint32_t)w));
}
constexpr int kPairs = 0xb1, kFours = 0x4e, kEights = 0x141, kSixteens = 0x140;
template <bool kHalves>
__device__ __forceinline__ void split(uint32_t w, uint32_t& even, uint32_t& odd) {
  const auto r = kHalves ? __builtin_amdgcn_permlane32_swap(w, w, false, false) : __builtin_amdgcn_permlane16_swap(w, w, false, false);
  even = r[0];
  odd = r[1];
}
template <bool kHalves>
__device__ __forceinline__ void split(float v, float& even, float& odd) {
  uint32_t a, b;
  split<kHalves>(__float_as_uint(v), a, b);
  even = __uint_as_float(a);
  odd = __uint_as_float(b);
}
template <bool kHalves>
__device__ __forceinline__ void split(double v, double& even, double& odd) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  uint32_t a0, b0, a1, b1;
  split<kHalves>((uint32_t)w, a0, b0);
  split<kHalves>((uint32_t)(w >> 32), a1, b1);
  even = __builtin_bit_cast(double, (uint64_t)a1 << 32 | a0);
  odd = __builtin_bit_cast(double, (uint64_t)b1 << 32 | b0);
}
template <typename T, typename F>
__device__ __forceinline__ T over_wave(T v, F join) {
  v = join(v, moved<kPairs>(v));
  v = join(v, moved<kFours>(v));
  v = join(v, moved<kEights>(v));
  v = join(v, moved<kSixteens>(v));
  T a, b;
  split<false>(v, a, b);
  v = join(a, b);
  split<true>(v, a, b);
  return join(a, b);
}
__device__ __forceinline__ float wave_max(float v) {
  return over_wave(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_sum(double v) {
  return over_wave(v, [](double a, double b) { return a + b; });
}

}  // namespace lg
}  // namespace caddtree
