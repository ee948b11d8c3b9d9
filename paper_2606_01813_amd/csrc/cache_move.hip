// The 4-bit cache's write and read: 16-bit tokens to codes and scales of their slots, and back.
//
// Both directions are bound by memory: 4 D bytes of 16-bit values and 1.0625 D of codes and scales a token
// and head.  A lane has 8 channels of keys and of values, 16 bytes, and four lanes a block of 32, so that
// neighbouring lanes read and write neighbouring pieces on either side.  Writing 4 x 4096 tokens of 8 heads of 128
// channels takes 17 us (85 MB, 5.0 TB/s), reading them back 15 us (5.7 TB/s).
#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kThreads = 256, kItems = 4;

// The scale's byte and the codes of a lane's 8 values (4 pairs) of a block that lanes 4 n .. 4 n + 3 hold.
// E = floor(log2 m) - 2 for the largest magnitude m, one more above 1.75 x 2^floor(log2 m); the hardware
// conversion rounds to the nearest code, ties to the even one, and saturates.
template <typename E>
__device__ uint32_t encode(const u32x4 x, uint32_t* scale_byte) {
  uint32_t top = 0;                                 // magnitudes order as integers, NaN above infinity
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fff, (x[i] >> 16) & 0x7fff));
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if (top >= E::kInf) {
    *scale_byte = 255;
    return 0;
  }
  const uint32_t f = __builtin_bit_cast(uint32_t, E::lo(top));   // (fp32: F16's subnormals are normal there)
  int e = (int)(f >> 23) - 127 - 2 + ((f & 0x7fffff) > 0x600000 ? 1 : 0);
  e = min(max(e, E::kExpLo), E::kExpHi);
  *scale_byte = (uint32_t)(e + 127);
  const float s = scale_of(e + 127);
  uint32_t r = 0;
  r = E::template to4<0>(r, x[0], s);
  r = E::template to4<1>(r, x[1], s);
  r = E::template to4<2>(r, x[2], s);
  r = E::template to4<3>(r, x[3], s);
  return r;
}

// A thread's token and head: rows of D / 8 lanes, heads innermost; the u-th of the n blocks of rows that a workgroup has.
struct Item {
  int t, h;
};
template <int D>
__device__ Item item_of(int heads, int u, int n) {
  constexpr int kPer = D / 8, kRows = kThreads / kPer;
  const uint32_t row = (blockIdx.x * n + u) * kRows + threadIdx.x / kPer;
  return Item{(int)(row / (uint32_t)heads), (int)(row % (uint32_t)heads)};
}

template <typename E, int D>
__global__ __launch_bounds__(kThreads) void write_kernel(CacheMoveArgs a) {
  using L = PageLayout<D>;
  const Item it = item_of<D>(a.kv.heads, 0, 1);
  const int b = blockIdx.y, piece = threadIdx.x % (D / 8);
  if (it.t >= (a.count ? clamp_len(a.count[b], a.T) : a.T)) return;      // (a block's four lanes stay together)
  const int64_t slot = a.start[b] + it.t;
  if (slot < 0 || slot >= (int64_t)a.kv.table_pages * kPage) return;
  int row = it.t;
  if (a.index) {
    row = a.index[(int64_t)b * a.T + it.t];
    if (row < 0 || row >= a.rows) return;
  }
  uint8_t* page = page_of(a.kv, b, (int)(slot / kPage), it.h);
  if (page == nullptr) return;
  const int tok = (int)(slot % kPage);
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.k.data + 2 * (b * a.k.b + row * a.k.t + it.h * a.k.h + piece * 8));
  const u32x4 v = *reinterpret_cast<const u32x4*>(a.v.data + 2 * (b * a.v.b + row * a.v.t + it.h * a.v.h + piece * 8));
  uint32_t ks, vs;
  const uint32_t kc = encode<E>(k, &ks), vc = encode<E>(v, &vs);
  *reinterpret_cast<uint32_t*>(page + L::kK + tok * L::kRow + piece * 4) = kc;
  *reinterpret_cast<uint32_t*>(page + L::kV + tok * L::kRow + piece * 4) = vc;
  if (piece % 4 == 0) {
    page[L::kKs + tok * L::kScales + piece / 4] = (uint8_t)ks;
    page[L::kVs + tok * L::kScales + piece / 4] = (uint8_t)vs;
  }
}

template <typename E>
__device__ u32x4 decode(uint32_t codes, uint32_t scale_byte) {
  if (scale_byte == 255) return u32x4{E::kNaN, E::kNaN, E::kNaN, E::kNaN};
  const float s = scale_of(scale_byte);
  return u32x4{E::template from4<0>(codes, s), E::template from4<1>(codes, s), E::template from4<2>(codes, s),
               E::template from4<3>(codes, s)};
}

// (kItems rows a thread, their loads in flight together: 131k tokens of 8 heads in 140 us, 4.9 TB/s, where one row a
// thread takes 162; writing gains nothing by it)
template <typename E, int D>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheMoveArgs a) {
  using L = PageLayout<D>;
  const int b = blockIdx.y, piece = threadIdx.x % (D / 8);
  const int64_t start = a.start ? a.start[b] : 0, end = min(a.end[b], (int64_t)a.kv.table_pages * kPage);
  bool there[kItems];
  uint32_t kc[kItems], vc[kItems], ks[kItems], vs[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const Item it = item_of<D>(a.kv.heads, u, kItems);
    const int64_t slot = start + it.t;
    there[u] = it.t < a.T && slot >= 0 && slot < end;
    if (!there[u]) continue;
    const uint8_t* page = page_of(a.kv, b, (int)(slot / kPage), it.h);
    there[u] = page != nullptr;
    if (!there[u]) continue;
    const int tok = (int)(slot % kPage);
    kc[u] = *reinterpret_cast<const uint32_t*>(page + L::kK + tok * L::kRow + piece * 4);
    vc[u] = *reinterpret_cast<const uint32_t*>(page + L::kV + tok * L::kRow + piece * 4);
    ks[u] = page[L::kKs + tok * L::kScales + piece / 4];
    vs[u] = page[L::kVs + tok * L::kScales + piece / 4];
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    if (!there[u]) continue;
    const Item it = item_of<D>(a.kv.heads, u, kItems);
    *reinterpret_cast<u32x4*>(a.k.data + 2 * (b * a.k.b + it.t * a.k.t + it.h * a.k.h + piece * 8)) = decode<E>(kc[u], ks[u]);
    *reinterpret_cast<u32x4*>(a.v.data + 2 * (b * a.v.b + it.t * a.v.t + it.h * a.v.h + piece * 8)) = decode<E>(vc[u], vs[u]);
  }
}

dim3 grid_of(const CacheMoveArgs& a, int D, int items) {
  const int64_t rows = items * kThreads / (D / 8);
  return dim3((unsigned)(((int64_t)a.T * a.kv.heads + rows - 1) / rows), a.B);
}

}  // namespace

hipError_t launch_cache_write(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g = grid_of(a, D, 1);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) write_kernel<BF16, 64><<<g, kThreads, 0, stream>>>(a);
    else write_kernel<BF16, 128><<<g, kThreads, 0, stream>>>(a);
  } else {
    if (D == 64) write_kernel<F16, 64><<<g, kThreads, 0, stream>>>(a);
    else write_kernel<F16, 128><<<g, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g = grid_of(a, D, kItems);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) read_kernel<BF16, 64><<<g, kThreads, 0, stream>>>(a);
    else read_kernel<BF16, 128><<<g, kThreads, 0, stream>>>(a);
  } else {
    if (D == 64) read_kernel<F16, 64><<<g, kThreads, 0, stream>>>(a);
    else read_kernel<F16, 128><<<g, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace caddtree
