// Attention over the keys of a tensor or of a 4-bit cache: one wavefront a query and head.
//
// Lanes are keys for the scores and channels for the sum over values; a running maximum and sum carry
// the softmax over tiles of 64 keys.  Keys that a row does not see are never read for it.
#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

// one row's state: channels lane, lane + 64
template <int D>
struct Row {
  float m = -INFINITY, l = 0.f, acc[D / 64] = {};
};

// keys of a tile of 64: lane's score (or -inf where it is not seen), then the values of the seen ones
template <typename E, int D, typename ValueOf>
__device__ void take(Row<D>& r, float s, ValueOf value) {
  float m = s;
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const uint64_t seen = __ballot(s != -INFINITY);       // (a NaN is seen)
  if (seen == 0) return;
  m = fmaxf(m, r.m);
  const float was = r.m == -INFINITY ? 0.f : __expf(r.m - m);
  const float p = s == -INFINITY ? 0.f : __expf(s - m);
  float l = p;
#pragma unroll
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  r.l = r.l * was + l;
  r.m = m;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) r.acc[c] *= was;
  for (uint64_t left = seen; left; left &= left - 1) {
    const int j = __builtin_ctzll(left);
    const float pj = __shfl(p, j);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) r.acc[c] += pj * value(j, c);
  }
}

template <typename E>
__device__ float dot(const char* q, const char* k, int D) {
  float s = 0.f;
  for (int d = 0; d < D; d += 2) {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(q + 2 * d), y = *reinterpret_cast<const uint32_t*>(k + 2 * d);
    s += E::lo(x) * E::lo(y);
    s += E::hi(x) * E::hi(y);
  }
  return s;
}

template <typename E, int D>
__global__ __launch_bounds__(64) void attention_kernel(AttnArgs a) {
  using L = PageLayout<D>;
  const int lane = threadIdx.x, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, hk = h / a.G;
  const Seq s = sequence(a, b);
  if (i >= s.nq) return;
  const int pos = s.base + step(a, b, i);
  const char* q = a.q.data + 2 * (b * a.q.b + i * a.q.t + h * a.q.h);
  Row<D> r;
  for (int t = 0; t < s.ctx; t += 64) {
    const int p = t + lane;
    const uint8_t* page = page_of(a.kv, b, t / kPage, hk);
    float x = -INFINITY;
    if (page && p < s.ctx && in_window(a, pos, p)) {
      x = 0.f;
      for (int blk = 0; blk < D / kBlock; ++blk) {
        uint32_t y[16];
        decode_block<E>(*reinterpret_cast<const u32x4*>(page + L::kK + lane * L::kRow + blk * 16),
                        page[L::kKs + lane * L::kScales + blk], y);
        for (int w = 0; w < 16; ++w) {
          const uint32_t z = *reinterpret_cast<const uint32_t*>(q + 2 * (blk * kBlock + 2 * w));
          x += E::lo(z) * E::lo(y[w]);
          x += E::hi(z) * E::hi(y[w]);
        }
      }
      x *= a.scale;
    }
    take<E, D>(r, x, [&](int j, int c) {
      const int d = lane + 64 * c;
      const uint8_t sc = page[L::kVs + j * L::kScales + d / kBlock];
      const uint32_t y = sc == 255 ? E::kNaN : E::template from4<0>(page[L::kV + j * L::kRow + d / 2], scale_of(sc));
      return d & 1 ? E::hi(y) : E::lo(y);
    });
  }
  for (int t = 0; t < s.nk; t += 64) {
    const int j = t + lane;
    float x = -INFINITY;
    if (j < s.nk) {
      const int pj = (a.kv.pages ? s.base : 0) + step(a, b, j);
      bool seen = in_window(a, pos, pj);
      if (a.order == CADDTREE_ORDER_CHAIN) seen = seen && pj <= pos;
      if (a.order == CADDTREE_ORDER_TREE) seen = seen && tree_sees(a, b, i, j);
      if (seen) x = a.scale * dot<E>(q, a.k.data + 2 * (b * a.k.b + j * a.k.t + hk * a.k.h), D);
    }
    take<E, D>(r, x, [&](int jj, int c) {
      const uint16_t v = *reinterpret_cast<const uint16_t*>(a.v.data + 2 * (b * a.v.b + (t + jj) * a.v.t + hk * a.v.h + lane + 64 * c));
      return E::lo(v);
    });
  }
  uint16_t* o = reinterpret_cast<uint16_t*>(a.out.data + 2 * (b * a.out.b + i * a.out.t + h * a.out.h));
  for (int c = 0; c < D / 64; ++c) o[lane + 64 * c] = (uint16_t)E::pair(r.m == -INFINITY ? 0.f : r.acc[c] / r.l, 0.f);
  if (a.lse && lane == 0) a.lse[((int64_t)b * a.T + i) * a.Hq + h] = r.m == -INFINITY ? -INFINITY : r.m + __logf(r.l);
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g(a.T, a.Hq, a.B);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) attention_kernel<BF16, 64><<<g, 64, 0, stream>>>(a);
    else attention_kernel<BF16, 128><<<g, 64, 0, stream>>>(a);
  } else {
    if (D == 64) attention_kernel<F16, 64><<<g, 64, 0, stream>>>(a);
    else attention_kernel<F16, 128><<<g, 64, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace caddtree
