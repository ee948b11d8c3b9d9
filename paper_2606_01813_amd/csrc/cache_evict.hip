// Eviction: which slots a kv head keeps (the sinks, the recent ones, and the largest scores of the
// rest), and the move of their codes, scales and scores to the new pages.
//
// Selection is a radix search for the smallest kept score: scores as order-preserving 32-bit keys, a
// histogram of 8 bits a pass, then one ordered pass that lists the kept slots.  Counts are integers,
// so nothing depends on the order of the additions.  One workgroup a sequence and kv head.
#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// order-preserving: larger scores, larger keys; -0 as 0, a NaN below everything
__device__ uint32_t key_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ int live_slots(const EvictArgs& a, int b) {
  return clamp_len(a.ctx_len[b], min((int64_t)a.kv.table_pages * kPage, a.slots));
}

__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kWaves][256];
  __shared__ uint32_t total[256];
  __shared__ uint32_t chosen[2];                    // the digit, and how many keys lie above it
  __shared__ uint32_t above[kWaves], equal[kWaves];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int n = live_slots(a, b), m = min(n, a.budget);
  int32_t* kept = a.kept + ((int64_t)b * a.kv.heads + h) * a.budget;
  const float* x = a.scores + ((int64_t)b * a.kv.heads + h) * a.slots;
  if (h == 0 && tid == 0) a.new_len[b] = m;
  for (int i = m + tid; i < a.budget; i += kThreads) kept[i] = -1;
  if (n <= a.budget) {
    for (int i = tid; i < n; i += kThreads) kept[i] = i;
    return;
  }
  // slots lo .. hi - 1 compete for `want` places (the sinks and the recent ones leave room for them)
  const int lo = a.sinks, hi = n - a.recent;
  uint32_t want = (uint32_t)(m - a.sinks - a.recent);
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < kWaves * 256; i += kThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kThreads) {
      const uint32_t k = key_of(x[i]);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[wave][(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t s = 0;
      for (int w = 0; w < kWaves; ++w) s += hist[w][tid];
      total[tid] = s;
    }
    __syncthreads();
    if (tid == 0) {
      // the digit whose keys hold the want-th largest; want = 0 ends at the top digit with none above
      uint32_t over = 0;
      int d = 255;
      while (d > 0 && over + total[d] < want) over += total[d--];
      chosen[0] = (uint32_t)d;
      chosen[1] = over;
    }
    __syncthreads();
    prefix |= chosen[0] << shift;
    want -= chosen[1];
    __syncthreads();
  }
  // kept: keys above prefix, and the first `want` equal to it.  A wavefront lists a strip of its own.
  const int strip = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int from = min(wave * strip, n), to = min(from + strip, n);
  auto kind = [&](int i) -> int {                   // 2 kept, 1 equal, 0 not kept
    if (i < lo || i >= hi) return 2;
    const uint32_t k = key_of(x[i]);
    return k > prefix ? 2 : k == prefix ? 1 : 0;
  };
  uint32_t na = 0, ne = 0;
  for (int t = from; t < to; t += 64) {
    const int i = t + lane, k = i < to ? kind(i) : 0;
    na += __popcll(__ballot(k == 2));
    ne += __popcll(__ballot(k == 1));
  }
  if (lane == 0) {
    above[wave] = na;
    equal[wave] = ne;
  }
  __syncthreads();
  uint32_t at = 0, eq = 0;                          // places taken and equal keys seen before this strip
  for (int w = 0; w < wave; ++w) {
    at += above[w] + (min(eq + equal[w], want) - min(eq, want));
    eq += equal[w];
  }
  const uint64_t below = (1ull << lane) - 1;
  for (int t = from; t < to; t += 64) {
    const int i = t + lane, k = i < to ? kind(i) : 0;
    const uint64_t eqs = __ballot(k == 1);
    const bool take = k == 2 || (k == 1 && eq + __popcll(eqs & below) < want);
    const uint64_t takes = __ballot(take);
    if (take) kept[at + __popcll(takes & below)] = i;
    at += __popcll(takes);
    eq += __popcll(eqs);
  }
}

// one token is D / 16 lanes' (16 bytes of codes each, keys then values); the first of each half also
// moves the scales
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a) {
  const int D = a.head_dim, per = D / 16, h = blockIdx.y, b = blockIdx.z;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / per;
  const int piece = threadIdx.x % per;
  const int64_t most = max((int64_t)a.budget, a.new_slots);
  if (i >= most) return;
  const int n = live_slots(a, b), m = min(n, a.budget);
  const int64_t row = (int64_t)b * a.kv.heads + h;
  if (i >= m) {
    if (piece == 0 && i < a.new_slots) a.new_scores[row * a.new_slots + i] = 0.f;
    return;
  }
  const int src = a.kept[row * a.budget + i];
  if (src < 0 || src >= n) return;
  if (piece == 0 && i < a.new_slots) a.new_scores[row * a.new_slots + i] = a.scores[row * a.slots + src];
  PagedKV to = a.kv;
  to.table = a.new_table;
  to.table_pages = a.new_pages;
  const uint8_t* from = page_of(a.kv, b, src / kPage, h);
  uint8_t* dst = page_of(to, b, (int)(i / kPage), h);
  if (from == nullptr || dst == nullptr) return;
  const int s = src % kPage, d = (int)(i % kPage), half = per / 2, row_bytes = D / 2, scales = D / kBlock;
  const int codes = piece < half ? 0 : kPage * row_bytes, at = piece % half * 16;
  *reinterpret_cast<u32x4*>(dst + codes + d * row_bytes + at) =
      *reinterpret_cast<const u32x4*>(from + codes + s * row_bytes + at);
  if (at == 0) {
    const int base = 2 * kPage * row_bytes + (piece < half ? 0 : kPage * scales);
    if (scales == 4)
      *reinterpret_cast<uint32_t*>(dst + base + 4 * d) = *reinterpret_cast<const uint32_t*>(from + base + 4 * s);
    else
      *reinterpret_cast<uint16_t*>(dst + base + 2 * d) = *reinterpret_cast<const uint16_t*>(from + base + 2 * s);
  }
}

}  // namespace

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
  select_kernel<<<dim3(a.kv.heads, a.B), kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t most = a.budget > a.new_slots ? a.budget : a.new_slots;
  if (most == 0) return hipSuccess;
  move_kernel<<<dim3((unsigned)((most * (a.head_dim / 16) + 255) / 256), a.kv.heads, a.B), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace caddtree
