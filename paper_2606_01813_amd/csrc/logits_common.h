// Device code shared by the kernels on logits: element types, vectors of 16 bytes at any element's address, sums.
#pragma once

#include <hip/hip_runtime.h>

#include "logits_args.h"

namespace caddtree {
namespace lg {

constexpr int kWave = 64;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// An element type: kN elements in 16 bytes, to and from fp32 (to: rounded to the nearest, ties to even).
struct BF16 {
  using T = __bf16;
};
struct F16 {
  using T = _Float16;
};
struct F32 {
  using T = float;
};
template <typename E>
constexpr int kN = 16 / (int)sizeof(typename E::T);

// 16 bytes of elements.  Rows start at any element (a vocabulary or a stride of any length), so a vector is
// aligned to its elements alone; the hardware takes 16-byte loads and stores at such addresses.
template <typename E>
struct Packed {
  typedef typename E::T V __attribute__((ext_vector_type(kN<E>)));
  struct __attribute__((packed, aligned(sizeof(typename E::T)))) Loose {
    V v;
  };
  V v;
  static __device__ __forceinline__ Packed load(const typename E::T* p) {
    return Packed{reinterpret_cast<const Loose*>(p)->v};
  }
  __device__ __forceinline__ void store(typename E::T* p) const { reinterpret_cast<Loose*>(p)->v = v; }
  // the first n elements (n < kN at a row's end), zeros behind
  static __device__ __forceinline__ Packed load_some(const typename E::T* p, int n) {
    Packed r = {};
#pragma unroll
    for (int j = 0; j < kN<E>; ++j)
      if (j < n) r.v[j] = p[j];
    return r;
  }
  __device__ __forceinline__ void store_some(typename E::T* p, int n) const {
#pragma unroll
    for (int j = 0; j < kN<E>; ++j)
      if (j < n) p[j] = v[j];
  }
  __device__ __forceinline__ float operator[](int j) const { return (float)v[j]; }
  __device__ __forceinline__ void set(int j, float x) { v[j] = (typename E::T)x; }
};

template <typename E>
__device__ __forceinline__ typename E::T* row_of(const Rows& r, int64_t b, int64_t t) {
  return reinterpret_cast<typename E::T*>(r.data) + b * r.b + t * r.t;
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
