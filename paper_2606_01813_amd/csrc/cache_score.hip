// Accumulated attention weight: what each cached key gets from a call's queries, added to its score.
//
// Bound by reading the keys, 0.53 D bytes a key and kv head, while the rows are few.  A wavefront holds a
// page's 64 keys as operands of the matrix product S = Q K^T, which has a key's scores for 16 rows on the
// four lanes of that key; it goes over the rows, sums a lane's weights in registers and adds the four lanes
// at the end.  No two wavefronts add to one score and the order of a sum is fixed.  Queries of no weight
// (in a tree most: only the accepted path counts) are left out first.  Where there are pages enough a wavefront
// has several, the next one's codes on their way, and what is set up once serves all of them.  64 single tokens over
// 4096 to 8192 cached ones, 8 kv heads of 128 channels: 55 us (4.6 TB/s, vector units busy 74% of the time; with a page a
// wavefront and operands kept for further rows the call took 97 us in place of 64); 8 trees of 65 rows over windows of 4096 of 16384: 36 us, of which
// the gathering of rows and the chain of first loads are the most.
#include <algorithm>

#include "attn_tile.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kWaves = 4, kChunk = 512;             // wavefronts; queries gathered at a time

// kOne: 16 rows at most, set up once (and a page's operands need not be kept for others).
template <typename E, int D, bool kOne>
__global__ __launch_bounds__(64 * kWaves, kOne ? 4 : 3) void score_kernel(ScoreArgs a, int pages) {
  using L = PageLayout<D>;
  __shared__ int query[kChunk], position[kChunk];
  __shared__ float weight[kChunk];
  __shared__ int counts[kWaves];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int hk = blockIdx.y, b = blockIdx.z, G = a.at.G;
  const Seq s = sequence(a.at, b);
  // a page that is out of every query's reach (all of them are at ctx or later) is not read
  const int lo = a.at.window == 0 ? 0 : s.base - a.at.window + 1;
  const int first = (blockIdx.x * pages * kWaves + wave) * kPage;    // the wavefront's pages are kWaves apart
  auto page_for = [&](int p0) -> const uint8_t* {
    const bool read = p0 < s.ctx && (p0 + kPage > lo || p0 < a.at.sinks);
    return read ? page_at(a.at.kv, table_entry(a.at.kv, b, p0 / kPage), hk) : nullptr;
  };
  uint32_t kc[4][D / 32] = {}, ks[4] = {};          // codes of key 16 u + col, channels g D / 4 ..; their scale
  auto load = [&](const uint8_t* page) {
    if (page == nullptr) return;
    const uint32_t code = col * L::kRow + g * (D / 8), scale = col * L::kScales + g * (D / 4) / kBlock;
    const uint8_t* scales = page + L::kKs;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t* c = reinterpret_cast<const uint32_t*>(page + (code + 16 * u * L::kRow));
#pragma unroll
      for (int j = 0; j < D / 32; ++j) kc[u][j] = c[j];
      ks[u] = scales[scale + 16 * u * L::kScales];
    }
  };
  const uint8_t* page = page_for(first);
  load(page);

  // the queries of some weight of a chunk, in their order
  int n = 0;
  auto gather = [&](int q0) {
    n = 0;
    for (int t = 0; t < kChunk && q0 + t < s.nq; t += 64 * kWaves) {
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
  };
  // rows r0 .. r0 + 15 of the chunk: the operand (row col), and rows 4 g + e
  u32x4 q[D / 32];
  float base[4], w[4];
  int from[4];
  auto rows = [&](int r0, int R) {
    const int rq = min(r0 + col, R - 1), iq = query[rq / G], hq = hk * G + rq % G;
    const u32x4* src = reinterpret_cast<const u32x4*>(a.at.q.data + 2 * (b * a.at.q.b + iq * a.at.q.t + hq * a.at.q.h + g * (D / 4)));
#pragma unroll
    for (int j = 0; j < D / 32; ++j) q[j] = src[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = min(r0 + 4 * g + e, R - 1), at = r / G, h = hk * G + r % G;
      base[e] = a.at.lse[b * a.lse_b + query[at] * a.lse_t + h * a.lse_h] * kLog2e;
      w[e] = r0 + 4 * g + e < R ? weight[at] : 0.f;
      from[e] = a.at.window == 0 ? 0 : position[at] - a.at.window + 1;
    }
  };
  const bool one_chunk = s.nq <= kChunk;
  if (one_chunk) gather(0);
  if (kOne && n > 0) rows(0, n * G);
  const float c = a.at.scale * kLog2e;
  auto operand = [&](int u, u32x4 (&key)[D / 32]) {
    const float f = scale_of(ks[u]);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      key[j] = u32x4{E::template from4<0>(kc[u][j], f), E::template from4<1>(kc[u][j], f), E::template from4<2>(kc[u][j], f),
                     E::template from4<3>(kc[u][j], f)};
    if (ks[u] == 255) key[0][0] = E::kNaN;          // (one is enough for the key's scores)
  };
  auto score = [&](const u32x4 (&key)[D / 32]) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) x = Mfma<E>::m16(q[j], key[j], x);
    return x;
  };
  auto weigh = [&](int p, f32x4 x) {                // what the four rows give key p
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool seen = w[e] > 0.f && (p >= from[e] || p < a.at.sinks);
      sum += seen ? w[e] * __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -base[e])) : 0.f;
    }
    return sum;
  };

  for (int k = 0; k < pages; ++k) {
    const int p0 = first + k * kWaves * kPage;
    const bool there = page != nullptr;
    float sum[4] = {};
    page = k + 1 < pages ? page_for(p0 + kWaves * kPage) : nullptr;
    if constexpr (kOne) {
      f32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        u32x4 key[D / 32];
        operand(u, key);
        x[u] = score(key);
      }
      load(page);
      if (there && n > 0)
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[u] = weigh(p0 + 16 * u + col, x[u]);
    } else {
      u32x4 key[4][D / 32];
#pragma unroll
      for (int u = 0; u < 4; ++u) operand(u, key[u]);
      load(page);
      for (int q0 = 0; q0 < s.nq; q0 += kChunk) {
        if (!one_chunk) gather(q0);
        if (there)
          for (int r0 = 0; r0 < n * G; r0 += 16) {
            rows(r0, n * G);
#pragma unroll
            for (int u = 0; u < 4; ++u) sum[u] += weigh(p0 + 16 * u + col, score(key[u]));
          }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      sum[u] += __shfl_xor(sum[u], 16);
      sum[u] += __shfl_xor(sum[u], 32);
    }
    const int64_t p = p0 + lane;                    // lane (col, g): key 16 g + col
    if (p < a.slots) {
      const float mine = g == 0 ? sum[0] : g == 1 ? sum[1] : g == 2 ? sum[2] : sum[3];
      const int64_t at = ((int64_t)b * a.at.Hkv + hk) * a.slots + p;
      a.new_scores[at] = a.scores[at] + (there && p < s.ctx ? mine : 0.f);
    }
  }
}

}  // namespace

namespace {

template <typename E, int D>
hipError_t launch(const ScoreArgs& a, hipStream_t stream) {
  // pages of a wavefront: several where a call reads so many that its workgroups would come in many rounds (2048 are on
  // the card at a time)
  const int64_t all = (a.slots + kPage - 1) / kPage;
  int64_t reach = all;
  if (a.at.window > 0) reach = std::min(all, ((int64_t)a.at.window + a.at.sinks) / kPage + 2);
  const int64_t waves = reach * a.at.Hkv * a.at.B;
  const int pages = (int)std::max<int64_t>(1, std::min<int64_t>(4, waves / (kWaves * 2048)));
  const dim3 g((unsigned)((all + kWaves * pages - 1) / (kWaves * pages)), a.at.Hkv, a.at.B);
  if ((int64_t)a.at.T * a.at.G <= 16) score_kernel<E, D, true><<<g, 64 * kWaves, 0, stream>>>(a, pages);
  else score_kernel<E, D, false><<<g, 64 * kWaves, 0, stream>>>(a, pages);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_score(const ScoreArgs& a, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) return D == 64 ? launch<BF16, 64>(a, stream) : launch<BF16, 128>(a, stream);
  return D == 64 ? launch<F16, 64>(a, stream) : launch<F16, 128>(a, stream);
}

}  // namespace caddtree
