// Accumulated attention weight: what each cached key gets from a call's queries, added to its score.
//
// Bound by reading the keys, 0.53 D bytes a key and kv head, while the rows are few.  A wavefront holds a
// page's 64 keys as operands of the matrix product S = Q K^T, which has a key's scores for 16 rows on the
// four lanes of that key; it goes over the rows, sums a lane's weights in registers and adds the four lanes
// at the end.  No two wavefronts add to one score and the order of a sum is fixed.  Queries of no weight
// (in a tree most: only the accepted path counts) are left out first.
#include "attn_tile.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kWaves = 4, kChunk = 512;             // pages of a workgroup; queries gathered at a time

template <typename E, int D>
__global__ __launch_bounds__(64 * kWaves, 3) void score_kernel(ScoreArgs a) {
  using L = PageLayout<D>;
  __shared__ int query[kChunk], position[kChunk];
  __shared__ float weight[kChunk];
  __shared__ int counts[kWaves];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int hk = blockIdx.y, b = blockIdx.z, G = a.at.G;
  const Seq s = sequence(a.at, b);
  const int p0 = (blockIdx.x * kWaves + wave) * kPage;
  // out of every query's reach: all of them are at ctx or later
  const int lo = a.at.window == 0 ? 0 : s.base - a.at.window + 1;
  const uint8_t* page = p0 < s.ctx && (p0 + kPage > lo || p0 < a.at.sinks) ? page_of(a.at.kv, b, p0 / kPage, hk) : nullptr;

  u32x4 k[4][D / 32];                               // key 16 u + col, channels g D / 4 + 8 j ..
  if (page) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t* c = reinterpret_cast<const uint32_t*>(page + L::kK + (16 * u + col) * L::kRow + g * (D / 8));
      const uint32_t sc = page[L::kKs + (16 * u + col) * L::kScales + g * (D / 4) / kBlock];
      const float f = scale_of(sc);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const uint32_t w = c[j];
        k[u][j] = u32x4{E::template from4<0>(w, f), E::template from4<1>(w, f), E::template from4<2>(w, f), E::template from4<3>(w, f)};
        if (sc == 255) k[u][j] = u32x4{E::kNaN, E::kNaN, E::kNaN, E::kNaN};
      }
    }
  }
  float sum[4] = {};
  const float c = a.at.scale * kLog2e;
  for (int q0 = 0; q0 < s.nq; q0 += kChunk) {
    // the chunk's queries of some weight, in their order
    int n = 0;
    for (int t = 0; t < kChunk; t += 64 * kWaves) {
      const int i = q0 + t + tid;
      float w = 0.f;
      if (i < min(s.nq, q0 + kChunk)) w = a.weight ? a.weight[(int64_t)b * a.at.T + i] : 1.f;
      const uint64_t some = __ballot(w > 0.f);
      __syncthreads();
      if (lane == 0) counts[wave] = __popcll(some);
      __syncthreads();
      int at = n;
      for (int v = 0; v < kWaves; ++v) {
        if (v < wave) at += counts[v];
        n += counts[v];
      }
      if (w > 0.f) {
        at += __popcll(some & ((1ull << lane) - 1));
        query[at] = i;
        position[at] = s.base + step(a.at, b, i);
        weight[at] = w;
      }
    }
    __syncthreads();
    if (page) {
      const int R = n * G;
      for (int r0 = 0; r0 < R; r0 += 16) {
        const int rq = min(r0 + col, R - 1), iq = query[rq / G], hq = hk * G + rq % G;
        const u32x4* src = reinterpret_cast<const u32x4*>(a.at.q.data + 2 * (b * a.at.q.b + iq * a.at.q.t + hq * a.at.q.h + g * (D / 4)));
        u32x4 q[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) q[j] = src[j];
        float base[4], w[4];                        // rows r0 + 4 g + e
        int from[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = min(r0 + 4 * g + e, R - 1), at = r / G, h = hk * G + r % G;
          base[e] = a.at.lse[((int64_t)b * a.at.T + query[at]) * a.at.Hq + h] * kLog2e;
          w[e] = r0 + 4 * g + e < R ? weight[at] : 0.f;
          from[e] = a.at.window == 0 ? 0 : position[at] - a.at.window + 1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < D / 32; ++j) x = Mfma<E>::m16(q[j], k[u][j], x);
          const int p = p0 + 16 * u + col;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool seen = w[e] > 0.f && (p >= from[e] || p < a.at.sinks);
            sum[u] += seen ? w[e] * __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -base[e])) : 0.f;
          }
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    sum[u] += __shfl_xor(sum[u], 16);
    sum[u] += __shfl_xor(sum[u], 32);
  }
  const int64_t p = p0 + lane;                      // lane (col, g): key 16 g + col
  if (p < a.slots) {
    const float mine = g == 0 ? sum[0] : g == 1 ? sum[1] : g == 2 ? sum[2] : sum[3];
    const int64_t at = ((int64_t)b * a.at.Hkv + hk) * a.slots + p;
    a.new_scores[at] = a.scores[at] + (page && p < s.ctx ? mine : 0.f);
  }
}

}  // namespace

hipError_t launch_cache_score(const ScoreArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  const dim3 g((unsigned)((a.slots + kPage * kWaves - 1) / (kPage * kWaves)), a.at.Hkv, a.at.B);
  if (dtype == CADDTREE_BF16) {
    if (D == 64) score_kernel<BF16, 64><<<g, 64 * kWaves, 0, stream>>>(a);
    else score_kernel<BF16, 128><<<g, 64 * kWaves, 0, stream>>>(a);
  } else {
    if (D == 64) score_kernel<F16, 64><<<g, 64 * kWaves, 0, stream>>>(a);
    else score_kernel<F16, 128><<<g, 64 * kWaves, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace caddtree
