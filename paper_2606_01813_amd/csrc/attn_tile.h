// Device code of the attention kernels: which keys a tile of rows reads, which of them each row sees, and
// the layouts of keys and values in LDS.
//
// All of them form S^T = K Q^T and O^T = V^T P^T, so a lane holds one query row in both products: the
// scores' layout is the one the second product wants of its weights (the key index of a matrix
// instruction is a sum's, any order serves), and a row's maximum and sum are a lane's own but for the
// lanes that hold the same row.  V^T comes out of a row-major tile through the transposing LDS read.
#pragma once

#include "attn_common.h"

namespace caddtree {
namespace at {

template <typename E>
struct Mfma;
template <>
struct Mfma<BF16> {
  static __device__ f32x4 m16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ f32x16 m32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma<F16> {
  static __device__ f32x4 m16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ f32x16 m32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// A row's sums are rescaled when its maximum has risen by more than this (in powers of two): they grow by 2^8 at
// most in between, and most tiles spare the products with every sum.
constexpr float kLag = 8.f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Scores are kept unscaled, so that a weight is one fused multiply-add and one exp2: exp2(s c - base) with
// c > 0 (-inf c has to be -inf).  A negative scale goes into the signs of q, and a scale of zero is the smallest normal
// number: products s of bf16 inputs may be as large as the largest one.
__device__ inline float score_factor(float scale) { return fmaxf(fabsf(scale) * kLog2e, 0x1p-126f); }
__device__ inline u32x4 signed_queries(u32x4 q, float scale) {
  const uint32_t flip = scale < 0.f ? 0x80008000u : 0u;
  return u32x4{q[0] ^ flip, q[1] ^ flip, q[2] ^ flip, q[3] ^ flip};
}

// The tiles that queries i0 .. i1 read: cached ones [0, a) and [b, c) of kC slots, new ones [0, d) and
// [e, f) of kN keys (first the sinks, then the window or everything); n of them in this order.
struct Span {
  int a, b, c, d, e, f, n;
};
__device__ inline int ceil_div(int x, int y) { return (x + y - 1) / y; }

template <int kC, int kN>
__device__ Span span_of(const AttnArgs& a, const Seq& s, int i0, int i1) {
  const bool tree = a.order == CADDTREE_ORDER_TREE, paged = a.kv.pages != nullptr;
  Span t;
  t.a = t.b = t.d = t.e = 0;
  t.c = ceil_div(s.ctx, kC);
  const int lo_idx = paged ? i0 : s.base + i0, hi_idx = paged ? i1 : s.base + i1;
  const int hi = a.order == CADDTREE_ORDER_CHAIN ? max(0, min(hi_idx + 1, s.nk)) : s.nk;
  t.f = ceil_div(hi, kN);
  if (a.window != 0) {
    const int lo = max(0, s.base + (tree ? 0 : i0) - a.window + 1);
    t.a = ceil_div(min(a.sinks, s.ctx), kC);
    t.b = lo >= s.ctx ? t.a : max(lo / kC, t.a);
    t.c = lo >= s.ctx ? t.a : max(t.c, t.b);
    if (!tree) {
      const int lj = max(0, lo_idx - a.window + 1);
      t.d = ceil_div(max(0, min(a.sinks - s.ctx, hi)), kN);
      t.e = lj >= hi ? t.d : max(lj / kN, t.d);
      t.f = lj >= hi ? t.d : max(t.f, t.e);
    }
  }
  t.n = t.a + (t.c - t.b) + t.d + (t.f - t.e);
  return t;
}
// tile t of a span: its first slot or key; *cached
template <int kC, int kN>
__device__ int tile_of(const Span& s, int t, bool* cached) {
  *cached = true;
  if (t < s.a) return t * kC;
  t -= s.a;
  if (t < s.c - s.b) return (s.b + t) * kC;
  t -= s.c - s.b;
  *cached = false;
  return (t < s.d ? t : s.e + t - s.d) * kN;
}

// A query row: its query, its position, and the new key's index that its own place has.
struct RowAt {
  int i, pos, idx;
};
__device__ inline RowAt row_at(const AttnArgs& a, const Seq& s, int b, int i) {
  return RowAt{i, s.base + step(a, b, i), a.kv.pages ? i : s.base + i};
}

__device__ inline uint64_t below(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// Which of the 64 slots from p0 on, or new keys from j0 on, a row sees: bit k for the k-th.  (Nothing here passes 32 bits:
// the host bounds the lengths and drops a window that is longer than they are.  Comparing before subtracting, which would
// need no bounds, cost the kernels registers: 32 rows over a cache took 5% longer.)
struct Sees {
  int slots, from, sinks;       // of keys: below `slots`, and from `from` on or below `sinks`
  __device__ uint64_t at(int k0) const { return below(slots - k0) & (~below(from - k0) | below(sinks - k0)); }
};
__device__ inline Sees sees_cached(const AttnArgs& a, const Seq& s, const RowAt& r) {
  return Sees{s.ctx, a.window == 0 ? 0 : r.pos - a.window + 1, a.sinks};
}
__device__ inline Sees sees_new(const AttnArgs& a, const Seq& s, const RowAt& r) {   // (chains and blocks)
  return Sees{a.order == CADDTREE_ORDER_CHAIN ? min(s.nk, r.idx + 1) : s.nk, a.window == 0 ? 0 : r.idx - a.window + 1,
              a.sinks - s.ctx};
}
__device__ inline uint64_t sees_tree(const AttnArgs& a, const Seq& s, int b, const RowAt& r, int j0) {
  uint64_t v = 0;
  if (r.i > 0) {                                   // bit k: node j0 + k - 1 of the mask's row i - 1
    const int64_t row = (int64_t)b * a.cap + r.i - 1;
    const int end = min(s.nk - j0, 64);            // (nodes at or past the tree's end are not looked at)
    if (a.mask_kind == CADDTREE_MASK_U8) {
      const uint8_t* m = static_cast<const uint8_t*>(a.mask) + row * a.cap + j0 - 1;
      for (int k = j0 == 0 ? 1 : 0; k < end; ++k) v |= (uint64_t)(m[k] != 0) << k;
    } else {
      const int words = (a.cap + 31) / 32, w = j0 / 32;
      const uint32_t* m = static_cast<const uint32_t*>(a.mask) + row * words;
      v = w < words ? m[w] : 0;
      if (w + 1 < words) v |= (uint64_t)m[w + 1] << 32;
      v = v << 1 | (w > 0 ? m[w - 1] >> 31 : 0);
    }
  }
  if (j0 == 0) v |= 1;                             // the root
  v &= below(s.nk - j0);
  const int depth = r.pos - s.base;
  if (a.window != 0 && depth >= a.window) {        // ancestors further up than the window
    for (uint64_t left = v; left; left &= left - 1) {
      const int k = __builtin_ctzll(left), pk = s.base + step(a, b, j0 + k);
      if (!in_window(a, r.pos, pk)) v &= ~(1ull << k);
    }
  }
  return v;
}
// every query of i0 .. i1 sees all n keys of the tile
__device__ inline bool full_cached(const AttnArgs& a, const Seq& s, int i1, int p0, int n) {
  const int last = s.base + (a.order == CADDTREE_ORDER_TREE ? s.nq : i1);
  return p0 + n <= s.ctx && (a.window == 0 || p0 > last - a.window || p0 + n <= a.sinks);
}
__device__ inline bool full_new(const AttnArgs& a, const Seq& s, int i0, int i1, int j0, int n) {
  if (a.order == CADDTREE_ORDER_TREE) return false;
  const int off = a.kv.pages ? 0 : s.base;
  return j0 + n <= (a.order == CADDTREE_ORDER_CHAIN ? min(s.nk, off + i0 + 1) : s.nk) &&
         (a.window == 0 || j0 > off + i1 - a.window || j0 + n <= a.sinks - s.ctx);
}

// LDS layouts.  A row is a token's D channels; 16-byte pieces trade places by the row so that the lanes that
// access LDS together (eight of 16 bytes, sixteen of 8) meet no bank twice: keys are read 16 bytes a lane,
// eight rows side by side; values 8 bytes a lane, four rows by 32 bytes, through the transposing read; both
// are written 16 bytes a lane, either a row's pieces in turn or, from a page, a piece of every block of
// 2 (D = 128) or 4 rows.
template <int D>
__device__ int k_at(int row, int piece) {          // piece: 16 bytes
  if (D == 128) return row * 256 + ((((piece & 3) << 2 | piece >> 2) ^ ((row & 1) << 2 | ((row >> 1) & 3) | (row & 8))) << 4);
  return row * 128 + ((((piece & 3) << 1 | piece >> 2) ^ ((row & 3) << 1 | ((row >> 2) & 1))) << 4);
}
// keys 16 j channels further (two pieces a step) are at k_at ^ k_step(j)
template <int D>
__device__ constexpr int k_step(int j) {
  const int piece = 2 * j;
  return (D == 128 ? (piece & 3) << 2 | piece >> 2 : (piece & 3) << 1 | piece >> 2) << 4;
}
// the n-th piece of a row that is written piece after piece
template <int D>
__device__ int k_piece(int n) {
  return D == 128 ? (n & 3) << 2 | n >> 2 : n;
}
template <int D>
__device__ int v_at(int row, int byte) {
  const int block = byte >> 6, sub = (byte >> 4) & 3, y = row & 3;
  if (D == 128) return row * 256 + ((block ^ y) << 6) + ((sub ^ y ^ ((row >> 1) & 2) ^ (block & 2)) << 4) + (byte & 15);
  return row * 128 + ((block ^ (y & 1)) << 6) + ((sub ^ y) << 4) + (byte & 15);
}
// the piece that lies in 16-byte place n of a row: k_at(row, k_there(row, n)) = row's start + 16 n, and of v_at
template <int D>
__device__ int k_there(int row, int n) {
  if (D == 128) return k_piece<D>(n ^ ((row & 1) << 2 | ((row >> 1) & 3) | (row & 8)));
  const int m = n ^ ((row & 3) << 1 | ((row >> 2) & 1));
  return m >> 1 | (m & 1) << 2;
}
template <int D>
__device__ int v_there(int row, int n) {
  const int y = row & 3;
  if (D == 128) return ((n >> 2) ^ y) << 2 | ((n & 3) ^ y ^ ((row >> 1) & 2) ^ (((n >> 2) ^ y) & 2));
  return ((n >> 2) ^ (y & 1)) << 2 | ((n & 3) ^ y);
}
// values `byte` (a multiple of 32) bytes further are at v_at ^ v_step(byte)
__device__ constexpr int v_step(int byte) { return byte ^ ((byte >> 6) & 2) << 4; }

// the larger of the values of lanes l and l ^ 32, l ^ 16
__device__ inline float max_across_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t lo = r[0], hi = r[1];
  return fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}
__device__ inline float max_across_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t lo = r[0], hi = r[1];
  return fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
// four rows of one channel: lane l of 16 gives the address of row l / 4 and channels 4 (l % 4) .. + 3 and
// gets channel l's four rows
__device__ inline u32x2 read_transposed(const char* lds) {
  typedef __attribute__((address_space(3))) s16x4* P;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds)));
}

// Values that a row does not see must not meet its weights of zero (0 x NaN), so a tile that some row sees
// in part is staged with zeros for keys that are not there and for values that are not finite.  Where there
// were any of the latter, the tiles are gone over again at the end and they are added to the rows that see
// them: what is not finite outlasts any later rescaling, so it does not matter when it is added.
template <typename E>
__device__ bool clean_pairs(u32x4& x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & E::kInf) == E::kInf) {
      bad = true;
      x[i] &= 0xffff0000u;
    }
    if ((x[i] & (E::kInf << 16)) == (E::kInf << 16)) {
      bad = true;
      x[i] &= 0x0000ffffu;
    }
  }
  return bad;
}
// four channels of a value row, what is finite among them replaced by 0
template <typename E>
__device__ f32x4 unclean(const char* at) {
  const u32x2 x = *reinterpret_cast<const u32x2*>(at);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[2 * i] = (x[i] & E::kInf) == E::kInf ? E::lo(x[i]) : 0.f;
    v[2 * i + 1] = (x[i] & (E::kInf << 16)) == (E::kInf << 16) ? E::hi(x[i]) : 0.f;
  }
  return v;
}

}  // namespace at
}  // namespace caddtree
