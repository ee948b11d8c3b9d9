// Eviction: which slots a kv head keeps (the sinks, the recent ones, and the largest scores of the
// rest), and the move of their codes, scales and scores to the new pages.
//
// Selection finds the smallest kept score, as an order-preserving 32-bit key, digit by digit (11, 11 and 10
// bits): a histogram of the first digit over all scores; the keys of the digit that holds the threshold
// then fit LDS as a rule and the other digits are found there.  A last ordered pass lists the kept slots.
// Counts are integers, so nothing depends on the order of the additions.  One workgroup a sequence and
// kv head; up to 16 scores a thread stay in registers throughout, longer rows are read from the L2 again.
#include <algorithm>

#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048, kRoom = 8192;

// order-preserving: larger scores, larger keys; -0 as 0, a NaN below everything
__device__ uint32_t key_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ int live_slots(const EvictArgs& a, int b) {
  return clamp_len(a.ctx_len[b], min((int64_t)a.kv.table_pages * kPage, a.slots));
}

// Adds to hist[d] of every lane with `is`.  Scores repeat (zeros above all), so the digit of the first lane is
// added once for all lanes that have it.
__device__ void count_digit(uint32_t* hist, bool is, uint32_t d) {
  const uint64_t any = __ballot(is);
  if (any == 0) return;
  const uint32_t first = __builtin_amdgcn_readlane(d, __builtin_ctzll(any));
  const uint64_t same = __ballot(is && d == first);
  if (is && d != first) atomicAdd(&hist[d], 1u);
  if ((threadIdx.x & 63) == __builtin_ctzll(same)) atomicAdd(&hist[first], (uint32_t)__popcll(same));
}

// The digit that holds the want-th largest key, and how many keys lie in larger digits; hist is cleared.
// With want = 0 it is the top digit, with none above.
__device__ void find_digit(uint32_t* hist, uint32_t* sums, uint32_t* found, uint32_t want) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // thread t has the two digits that rank 2 t and 2 t + 1 from the top
  const int top = kBins - 1 - 2 * tid;
  const uint32_t c0 = hist[top], c1 = hist[top - 1];
  uint32_t s = c0 + c1;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)s, o);
    if (lane >= o) s += y;
  }
  if (lane == 63) sums[wave] = s;
  hist[top] = hist[top - 1] = 0;
  if (tid == 0) {
    found[0] = kBins - 1;
    found[1] = 0;
  }
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += sums[w];
  s += before;                                      // keys down to this thread's second digit
  const uint32_t above = s - c0 - c1;
  if (above < want && want <= s) {
    const bool second = above + c0 < want;
    found[0] = (uint32_t)(second ? top - 1 : top);
    found[1] = second ? above + c0 : above;
  }
  __syncthreads();
}

// kKept: keys a thread holds (kKept kThreads >= n), or 0: scores are read again each time
template <int kKept>
__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t room[kKept ? 1 : kRoom];      // keys of the threshold's first digit
  __shared__ uint32_t sums[kWaves], equals[kWaves], found[2], filled;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
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
  // a wavefront has a strip of its own, 64 slots a step
  const int strip = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int from = min(wave * strip, n), to = min(from + strip, n);
  uint32_t mine[kKept ? kKept : 1];
  if (kKept)
#pragma unroll
    for (int j = 0; j < kKept; ++j) {
      const int i = from + 64 * j + lane;
      mine[j] = i < to ? key_of(x[i]) : 0;
    }
  // f(slot, key) for the lanes' slots of a strip, all lanes together; a slot past the strip is -1
  auto every = [&](auto f) {
    if constexpr (kKept != 0) {
#pragma unroll
      for (int j = 0; j < kKept; ++j)
        if (from + 64 * j < to) {
          const int i = from + 64 * j + lane;
          f(i < to ? i : -1, mine[j]);
        }
    } else {
      for (int t = from; t < to; t += 512) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = t + 64 * j + lane;
          y[j] = i < to ? x[i] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (t + 64 * j < to) {
            const int i = t + 64 * j + lane;
            f(i < to ? i : -1, key_of(y[j]));
          }
      }
    }
  };
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  if (tid == 0) filled = 0;
  __syncthreads();
  every([&](int i, uint32_t k) { count_digit(hist, i >= lo && i < hi, k >> 21); });
  __syncthreads();
  find_digit(hist, sums, found, want);
  uint32_t prefix = found[0] << 21;
  want -= found[1];
  bool fits = kKept == 0;
  if (kKept == 0) {                                 // the keys of this digit, where they fit
    every([&](int i, uint32_t k) {
      const bool is = i >= lo && i < hi && k >> 21 == prefix >> 21;
      const uint64_t some = __ballot(is);
      if (some == 0) return;
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&filled, (uint32_t)__popcll(some));
      at = __builtin_amdgcn_readfirstlane(at) + __popcll(some & ((1ull << lane) - 1));
      if (is && at < kRoom) room[at] = k;
    });
    __syncthreads();
    fits = filled <= kRoom;
  }
  for (int pass = 0; pass < 2; ++pass) {
    const int shift = pass == 0 ? 10 : 0, done = pass == 0 ? 21 : 10;
    const uint32_t mask = pass == 0 ? 2047 : 1023;
    if (fits) {
      const int c = (int)filled;
      for (int i = tid; i < (c + 63) / 64 * 64; i += kThreads) {
        const uint32_t k = i < c ? room[i] : 0;
        count_digit(hist, i < c && k >> done == prefix >> done, (k >> shift) & mask);
      }
    } else {
      every([&](int i, uint32_t k) { count_digit(hist, i >= lo && i < hi && k >> done == prefix >> done, (k >> shift) & mask); });
    }
    __syncthreads();
    if (want == 0) prefix |= mask << shift;          // (only where the sinks and the recent ones fill the budget)
    find_digit(hist, sums, found, want);
    if (want != 0) {
      prefix |= found[0] << shift;
      want -= found[1];
    }
  }
  // kept: keys above prefix, and the first `want` equal to it
  auto kind = [&](int i, uint32_t k) -> int {       // 2 kept, 1 equal, 0 not kept
    if (i < 0) return 0;
    if (i < lo || i >= hi) return 2;
    return k > prefix ? 2 : k == prefix ? 1 : 0;
  };
  uint32_t na = 0, ne = 0;
  every([&](int i, uint32_t k) {
    const int t = kind(i, k);
    na += __popcll(__ballot(t == 2));
    ne += __popcll(__ballot(t == 1));
  });
  if (lane == 0) {
    sums[wave] = na;
    equals[wave] = ne;
  }
  __syncthreads();
  uint32_t at = 0, eq = 0;                          // places taken and equal keys seen before this strip
  for (int w = 0; w < wave; ++w) {
    at += sums[w] + (min(eq + equals[w], want) - min(eq, want));
    eq += equals[w];
  }
  const uint64_t below = (1ull << lane) - 1;
  every([&](int i, uint32_t k) {
    const int t = kind(i, k);
    const uint64_t eqs = __ballot(t == 1);
    const bool take = t == 2 || (t == 1 && eq + __popcll(eqs & below) < want);
    const uint64_t takes = __ballot(take);
    if (take) kept[at + __popcll(takes & below)] = i;
    at += __popcll(takes);
    eq += __popcll(eqs);
  });
}

// A wavefront moves the 64 tokens of a new page and head: a lane looks up one token's old place, then
// D / 16 lanes move a token's codes, 16 bytes each, all loads in flight at once.
template <int D>
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a) {
  using L = PageLayout<D>;
  constexpr int kPer = D / 16, kSteps = kPer;       // lanes a token; steps of 64 / kPer tokens
  const int lane = threadIdx.x & 63, h = blockIdx.y, b = blockIdx.z;
  const int page = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = (int64_t)b * a.kv.heads + h, i = (int64_t)page * kPage + lane;
  const int n = live_slots(a, b), m = min(n, a.budget);
  int src = -1;
  if (i < m) src = a.kept[row * a.budget + i];
  if (src >= n) src = -1;
  if (i < a.new_slots) a.new_scores[row * a.new_slots + i] = src >= 0 ? a.scores[row * a.slots + src] : 0.f;
  if (page >= a.new_pages || (int64_t)page * kPage >= m) return;
  PagedKV to = a.kv;
  to.table = a.new_table;
  to.table_pages = a.new_pages;
  uint8_t* dst = page_of(to, b, page, h);
  const uint8_t* from = src >= 0 ? page_of(a.kv, b, src / kPage, h) : nullptr;
  if (dst == nullptr) return;
  const int tok = src % kPage;
  const uint64_t old = from ? reinterpret_cast<uint64_t>(from + tok * L::kRow) : 0;      // 0: nothing to move
  u32x4 x[kSteps];
  const int piece = lane % kPer, half = kPer / 2, at = (piece < half ? L::kK : L::kV) + piece % half * 16;
  uint32_t there = 0;
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int token = u * (64 / kPer) + lane / kPer;
    const uint64_t p = (uint64_t)(uint32_t)__shfl((int)(old >> 32), token) << 32 | (uint32_t)__shfl((int)old, token);
    // (nothing to move: the new place itself is read, and not written)
    x[u] = *reinterpret_cast<const u32x4*>((p ? p : reinterpret_cast<uint64_t>(dst) + token * L::kRow) + at);
    there |= (uint32_t)(p != 0) << u;
  }
  uint32_t ks = 0, vs = 0;
  if (from) {
    if (D == 128) {
      ks = *reinterpret_cast<const uint32_t*>(from + L::kKs + tok * 4);
      vs = *reinterpret_cast<const uint32_t*>(from + L::kVs + tok * 4);
    } else {
      ks = *reinterpret_cast<const uint16_t*>(from + L::kKs + tok * 2);
      vs = *reinterpret_cast<const uint16_t*>(from + L::kVs + tok * 2);
    }
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u)
    if ((there >> u) & 1) *reinterpret_cast<u32x4*>(dst + (u * (64 / kPer) + lane / kPer) * L::kRow + at) = x[u];
  if (from) {
    if (D == 128) {
      *reinterpret_cast<uint32_t*>(dst + L::kKs + lane * 4) = ks;
      *reinterpret_cast<uint32_t*>(dst + L::kVs + lane * 4) = vs;
    } else {
      *reinterpret_cast<uint16_t*>(dst + L::kKs + lane * 2) = (uint16_t)ks;
      *reinterpret_cast<uint16_t*>(dst + L::kVs + lane * 2) = (uint16_t)vs;
    }
  }
}

}  // namespace

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t stream) {
  const int64_t most = std::min<int64_t>((int64_t)a.kv.table_pages * kPage, a.slots);
  const dim3 g(a.kv.heads, a.B);
  // a strip is whole steps of 64, so a thread holds n / 1024 keys, rounded up
  if (most <= 4 * kThreads) select_kernel<4><<<g, kThreads, 0, stream>>>(a);
  else if (most <= 16 * kThreads) select_kernel<16><<<g, kThreads, 0, stream>>>(a);
  else select_kernel<0><<<g, kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.new_slots == 0) return e;
  const dim3 mg((unsigned)((a.new_slots + 4 * kPage - 1) / (4 * kPage)), a.kv.heads, a.B);
  if (a.head_dim == 64) move_kernel<64><<<mg, 256, 0, stream>>>(a);
  else move_kernel<128><<<mg, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace caddtree
