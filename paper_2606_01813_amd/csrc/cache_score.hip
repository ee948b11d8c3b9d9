// Accumulated attention weight: what each cached key gets from a call's queries, added to its score.
//
// A wavefront holds 64 keys of a page, one a lane, and goes over the queries; no two wavefronts add to
// one score, and the queries' order is fixed.
#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

template <typename E, int D>
__global__ __launch_bounds__(64) void score_kernel(ScoreArgs a) {
  using L = PageLayout<D>;
  const int lane = threadIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const int64_t p = (int64_t)blockIdx.x * kPage + lane;
  const Seq s = sequence(a.at, b);
  float sum = 0.f;
  const uint8_t* page = (int64_t)blockIdx.x * kPage < s.ctx ? page_of(a.at.kv, b, blockIdx.x, hk) : nullptr;
  if (page && p < s.ctx) {
    uint32_t y[D / 2];
    for (int blk = 0; blk < D / kBlock; ++blk)
      decode_block<E>(*reinterpret_cast<const u32x4*>(page + L::kK + lane * L::kRow + blk * 16),
                      page[L::kKs + lane * L::kScales + blk], y + 16 * blk);
    for (int i = 0; i < s.nq; ++i) {
      const float w = a.weight ? a.weight[(int64_t)b * a.at.T + i] : 1.f;
      if (!(w > 0.f) || !in_window(a.at, s.base + step(a.at, b, i), (int)p)) continue;
      for (int g = 0; g < a.at.G; ++g) {
        const int h = hk * a.at.G + g;
        const char* q = a.at.q.data + 2 * (b * a.at.q.b + i * a.at.q.t + h * a.at.q.h);
        float x = 0.f;
        for (int d = 0; d < D / 2; ++d) {
          const uint32_t z = *reinterpret_cast<const uint32_t*>(q + 4 * d);
          x += E::lo(z) * E::lo(y[d]);
          x += E::hi(z) * E::hi(y[d]);
        }
        sum += w * __expf(x * a.at.scale - a.at.lse[((int64_t)b * a.at.T + i) * a.at.Hq + h]);
      }
    }
  }
  if (p < a.slots) {
    const int64_t at = ((int64_t)b * a.at.Hkv + hk) * a.slots + p;
    a.new_scores[at] = a.scores[at] + sum;
  }
}

}  // namespace

hipError_t launch_cache_score(const ScoreArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g((unsigned)((a.slots + kPage - 1) / kPage), a.at.Hkv, a.at.B);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) score_kernel<BF16, 64><<<g, 64, 0, stream>>>(a);
    else score_kernel<BF16, 128><<<g, 64, 0, stream>>>(a);
  } else {
    if (D == 64) score_kernel<F16, 64><<<g, 64, 0, stream>>>(a);
    else score_kernel<F16, 128><<<g, 64, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace caddtree
