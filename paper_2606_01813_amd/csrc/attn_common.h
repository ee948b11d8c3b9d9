// Device code shared by the attention and cache kernels: element types, a sequence's lengths and
// positions, visibility, and the 4-bit page format.
#pragma once

#include <hip/hip_runtime.h>

#include "attn_args.h"

namespace caddtree {
namespace at {

constexpr int kPage = CADDTREE_PAGE;
constexpr int kBlock = CADDTREE_KV_BLOCK;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The 16-bit element types: pairs in a 32-bit register, the 4-bit conversions (exact: a code times a
// power of two) and the range of the scales' exponents.  Weights of the softmax are exp2(x - m + kBias) with a
// maximum m that may lag up to 8 behind (kLag): 2^8 at most in bf16; in f16, whose normal numbers end at
// 2^-14, 2^14 at most, and a weight keeps its 11 bits down to 2^-20 of 2^m.
struct BF16 {
  using T = __bf16;
  static constexpr int kExpLo = -125, kExpHi = 125;
  static constexpr float kBias = 0.f;
  static constexpr uint32_t kInf = 0x7f80;            // exponent bits, all ones for NaN and infinities
  static constexpr uint32_t kNaN = 0x7fc07fc0;        // a pair
  static __device__ float lo(uint32_t p) { return __builtin_bit_cast(float, p << 16); }
  static __device__ float hi(uint32_t p) { return __builtin_bit_cast(float, p & 0xffff0000u); }
  static __device__ uint32_t pair(float a, float b) {
    bf16x2 v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
  }
  template <int kByte>
  static __device__ uint32_t from4(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
  }
  template <int kByte>
  static __device__ uint32_t to4(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, pair), scale, kByte);
  }
};
struct F16 {
  using T = _Float16;
  static constexpr int kExpLo = -13, kExpHi = 13;
  static constexpr float kBias = 6.f;
  static constexpr uint32_t kInf = 0x7c00;
  static constexpr uint32_t kNaN = 0x7e007e00;
  static __device__ float lo(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[0]; }
  static __device__ float hi(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[1]; }
  static __device__ uint32_t pair(float a, float b) {
    f16x2 v;
    v[0] = (_Float16)a;
    v[1] = (_Float16)b;
    return __builtin_bit_cast(uint32_t, v);
  }
  template <int kByte>
  static __device__ uint32_t from4(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kByte));
  }
  template <int kByte>
  static __device__ uint32_t to4(uint32_t old, uint32_t pair, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, pair), scale, kByte);
  }
};

// 2^(code - 127) for a scale byte of 1 .. 254
__device__ inline float scale_of(uint32_t code) { return __builtin_bit_cast(float, code << 23); }

// One sequence of a call.  With a cache the keys are its ctx slots at positions 0 .. ctx - 1 and then nk
// new ones; query and new key i are at ctx + step(i).  Without one there are only the nk given, key j at
// j, and query i is at base + i.
struct Seq {
  int ctx, nq, nk, base;
};
__device__ inline int clamp_len(int64_t n, int64_t most) { return (int)(n < 0 ? 0 : n > most ? most : n); }
__device__ inline Seq sequence(const AttnArgs& a, int b) {
  Seq s;
  const bool tree = a.order == CADDTREE_ORDER_TREE;
  s.nq = a.q_len ? clamp_len((int64_t)a.q_len[b] + (tree ? 1 : 0), a.T) : a.T;
  if (a.kv.pages) {
    s.ctx = clamp_len(a.ctx_len[b], (int64_t)a.kv.table_pages * kPage);
    s.nk = a.k.data ? s.nq : 0;
    s.base = s.ctx;
  } else {
    s.ctx = 0;
    s.nk = a.k_len ? clamp_len(a.k_len[b], a.S) : a.S;
    s.base = s.nk - s.nq;
  }
  return s;
}
__device__ inline int step(const AttnArgs& a, int b, int i) {
  return a.order == CADDTREE_ORDER_TREE ? (i == 0 ? 0 : a.depth[(int64_t)b * a.cap + i - 1]) : i;
}
__device__ inline bool in_window(const AttnArgs& a, int pos_q, int pos_k) {
  return a.window == 0 || pos_q - pos_k < a.window || pos_k < a.sinks;
}

// The page of a slot and kv head: null where the table names no page of the cache.
__device__ inline uint8_t* page_of(const PagedKV& kv, int b, int page, int h) {
  const int32_t p = kv.table[(int64_t)b * kv.table_pages + page];
  if (p < 0 || p >= kv.n_pages) return nullptr;
  return kv.pages + ((int64_t)p * kv.heads + h) * kv.page_bytes;
}
// ... in two steps for a page that all lanes look up together: its table entry, loaded ahead, and the pointer in
// scalar registers, so that a lane's loads need no more than its 32-bit offset.
__device__ inline int32_t table_entry(const PagedKV& kv, int b, int page) { return kv.table[(int64_t)b * kv.table_pages + page]; }
__device__ inline uint8_t* page_at(const PagedKV& kv, int32_t entry, int h) {
  const int32_t p = __builtin_amdgcn_readfirstlane(entry);
  return p < 0 || p >= kv.n_pages ? nullptr : kv.pages + ((int64_t)p * kv.heads + h) * kv.page_bytes;
}
// Offsets in a page and head of head dimension D.
template <int D>
struct PageLayout {
  static constexpr int kRow = D / 2, kScales = D / kBlock;     // bytes of a token's codes and scales
  static constexpr int kK = 0, kV = kPage * kRow, kKs = 2 * kPage * kRow, kVs = kKs + kPage * kScales;
};

// 32 codes of a block as 16 pairs (out[i]: channels 2 i, 2 i + 1)
template <typename E>
__device__ inline void decode_block(const u32x4 codes, uint32_t scale_byte, uint32_t out[16]) {
  const float s = scale_of(scale_byte);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    out[4 * w + 0] = E::template from4<0>(codes[w], s);
    out[4 * w + 1] = E::template from4<1>(codes[w], s);
    out[4 * w + 2] = E::template from4<2>(codes[w], s);
    out[4 * w + 3] = E::template from4<3>(codes[w], s);
  }
  if (__any(scale_byte == 255))                      // (rare: one branch in place of 16 selects)
#pragma unroll
    for (int i = 0; i < 16; ++i) out[i] = scale_byte == 255 ? E::kNaN : out[i];
}

}  // namespace at
}  // namespace caddtree
