// The 4-bit cache's write and read: 16-bit tokens to codes and scales of their slots, and back.
//
// A block of 32 channels is a lane's: 64 bytes of input, 16 of codes and one of scale, keys and values
// one after the other.  Both directions are bound by memory: 4 D bytes of 16-bit values and 1.0625 D of
// codes and scales a token and head.
#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

// The scale's exponent and the codes of 32 values (16 pairs).  E = floor(log2 m) - 2 for the largest
// magnitude m, one more above 1.75 x 2^floor(log2 m); the hardware conversion rounds to the nearest
// code, ties to the even one, and saturates.
template <typename E>
__device__ u32x4 encode_block(const uint32_t x[16], uint32_t* scale_byte) {
  uint32_t top = 0;                                 // magnitudes order as integers, NaN above infinity
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t a = x[i] & 0x7fff, b = (x[i] >> 16) & 0x7fff;
    top = max(top, max(a, b));
  }
  if (top >= E::kInf) {
    *scale_byte = 255;
    return u32x4{0, 0, 0, 0};
  }
  const uint32_t f = __builtin_bit_cast(uint32_t, E::lo(top));   // (fp32: F16's subnormals are normal there)
  int e = (int)(f >> 23) - 127 - 2 + ((f & 0x7fffff) > 0x600000 ? 1 : 0);
  e = min(max(e, E::kExpLo), E::kExpHi);
  *scale_byte = (uint32_t)(e + 127);
  const float s = scale_of(e + 127);
  u32x4 c;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t r = 0;
    r = E::template to4<0>(r, x[4 * w + 0], s);
    r = E::template to4<1>(r, x[4 * w + 1], s);
    r = E::template to4<2>(r, x[4 * w + 2], s);
    r = E::template to4<3>(r, x[4 * w + 3], s);
    c[w] = r;
  }
  return c;
}

// item -> (sequence, token, head, block), blocks innermost: the lanes of a wavefront read whole heads
struct Item {
  int b, t, h, blk;
};
template <int D>
__device__ Item item_of(int64_t i, int T, int heads) {
  constexpr int n = D / kBlock;
  Item it;
  it.blk = (int)(i % n);
  i /= n;
  it.h = (int)(i % heads);
  i /= heads;
  it.t = (int)(i % T);
  it.b = (int)(i / T);
  return it;
}

template <typename E, int D>
__global__ __launch_bounds__(256) void write_kernel(CacheMoveArgs a) {
  using L = PageLayout<D>;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.B * a.T * a.kv.heads * (D / kBlock)) return;
  const Item it = item_of<D>(i, a.T, a.kv.heads);
  if (it.t >= (a.count ? clamp_len(a.count[it.b], a.T) : a.T)) return;
  const int64_t slot = (a.start ? a.start[it.b] : 0) + it.t;
  if (slot < 0 || slot >= (int64_t)a.kv.table_pages * kPage) return;
  int row = it.t;
  if (a.index) {
    row = a.index[(int64_t)it.b * a.T + it.t];
    if (row < 0 || row >= a.rows) return;
  }
  uint8_t* page = page_of(a.kv, it.b, (int)(slot / kPage), it.h);
  if (page == nullptr) return;
  const int tok = (int)(slot % kPage);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const View& v = kv ? a.v : a.k;
    const u32x4* src = reinterpret_cast<const u32x4*>(v.data + 2 * (it.b * v.b + row * v.t + it.h * v.h + it.blk * kBlock));
    uint32_t x[16];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const u32x4 y = src[w];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * w + j] = y[j];
    }
    uint32_t s;
    const u32x4 c = encode_block<E>(x, &s);
    *reinterpret_cast<u32x4*>(page + (kv ? L::kV : L::kK) + tok * L::kRow + it.blk * 16) = c;
    page[(kv ? L::kVs : L::kKs) + tok * L::kScales + it.blk] = (uint8_t)s;
  }
}

template <typename E, int D>
__global__ __launch_bounds__(256) void read_kernel(CacheMoveArgs a) {
  using L = PageLayout<D>;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.B * a.T * a.kv.heads * (D / kBlock)) return;
  const Item it = item_of<D>(i, a.T, a.kv.heads);
  const int64_t slot = (a.start ? a.start[it.b] : 0) + it.t;
  if (slot < 0 || slot >= a.end[it.b] || slot >= (int64_t)a.kv.table_pages * kPage) return;
  const uint8_t* page = page_of(a.kv, it.b, (int)(slot / kPage), it.h);
  if (page == nullptr) return;
  const int tok = (int)(slot % kPage);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const View& v = kv ? a.v : a.k;
    const u32x4 c = *reinterpret_cast<const u32x4*>(page + (kv ? L::kV : L::kK) + tok * L::kRow + it.blk * 16);
    uint32_t x[16];
    decode_block<E>(c, page[(kv ? L::kVs : L::kKs) + tok * L::kScales + it.blk], x);
    u32x4* dst = reinterpret_cast<u32x4*>(v.data + 2 * (it.b * v.b + it.t * v.t + it.h * v.h + it.blk * kBlock));
#pragma unroll
    for (int w = 0; w < 4; ++w) dst[w] = u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
  }
}

dim3 grid_of(const CacheMoveArgs& a, int D) {
  return dim3((unsigned)(((int64_t)a.B * a.T * a.kv.heads * (D / kBlock) + 255) / 256));
}

}  // namespace

hipError_t launch_cache_write(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g = grid_of(a, D);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) write_kernel<BF16, 64><<<g, 256, 0, stream>>>(a);
    else write_kernel<BF16, 128><<<g, 256, 0, stream>>>(a);
  } else {
    if (D == 64) write_kernel<F16, 64><<<g, 256, 0, stream>>>(a);
    else write_kernel<F16, 128><<<g, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g = grid_of(a, D);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) read_kernel<BF16, 64><<<g, 256, 0, stream>>>(a);
    else read_kernel<BF16, 128><<<g, 256, 0, stream>>>(a);
  } else {
    if (D == 64) read_kernel<F16, 64><<<g, 256, 0, stream>>>(a);
    else read_kernel<F16, 128><<<g, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace caddtree
