// Eviction: which slots a kv head keeps (the sinks, the recent ones, and the largest scores of the
// rest), and the move of their codes, scales and scores to the new pages.
//
// Selection finds the smallest kept score, as an order-preserving 32-bit key, digit by digit (11, 11 and 10
// bits), by a histogram of the digit over the keys that share the digits found so far.  A last ordered pass
// lists the kept slots.  Counts are integers, so nothing depends on the order of the additions.
// Slots of a page that is not in the cache hold no key: they are left out, neither counted nor kept.  A wavefront's step
// is 64 slots, a page, so whether they are there is a bit for all of them.
// Rows of up to 16384 slots have a workgroup each and keep their keys in registers throughout.  Longer rows
// are cut into parts, a workgroup each: a launch a digit counts every part's keys, the next one adds the parts'
// histograms up, finds the digit and goes on, and the last lists (kept slots before a part follow from the
// histograms of the parts before it).  4 rows with the move: of 16384 slots 29 us in a workgroup, of 16448 32 us in
// parts; of 131072 34 us of selection in parts, 137 in a workgroup that reads its scores again for every digit.
// Bound by latency: a part's counting takes 5 us, adding the histograms 3 more (parts of 4096 or of 16384 slots: the
// whole call 46 -> 60 and 51 us).
#include <algorithm>

#include "attn_common.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
constexpr int kHeld = 16;                                    // keys a thread holds at most in select_kernel
constexpr int kStep = 8, kBlock = kStep * kThreads;          // slots a workgroup of the parts takes at a time

// order-preserving: larger scores, larger keys; -0 as 0, a NaN below everything
__device__ uint32_t key_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ int live_slots(const EvictArgs& a, int b) {
  return clamp_len(a.ctx_len[b], min((int64_t)a.kv.table_pages * kPage, a.slots));
}

// Lane j's page: of the 64 slots from i0 + 64 j on, where j < steps and they are below `to`; and which of them are there.
__device__ __forceinline__ int32_t entries(const EvictArgs& a, int b, int i0, int steps, int to) {
  const int lane = threadIdx.x & 63, i = i0 + 64 * lane;
  return lane < steps && i < to ? table_entry(a.kv, b, i / kPage) : -1;
}
__device__ __forceinline__ uint64_t pages_there(const EvictArgs& a, int32_t entry) { return __ballot(entry >= 0 && entry < a.kv.n_pages); }
// Of the slots i0 .. i1 - 1 those outside lo .. hi - 1, which do not compete.
__device__ __forceinline__ int outside(int i0, int i1, int lo, int hi) { return i1 - i0 - max(0, min(i1, hi) - max(i0, lo)); }
// Adds the slots from i0 on that are there to *slots, and those of them that do not compete to *fixed.
__device__ __forceinline__ void add_there(uint64_t there, int i0, int steps, int to, int lo, int hi, int* slots, int* fixed) {
  const int end = min(i0 + 64 * steps, to), n = max(0, (end - i0 + 63) / 64);
  if ((int)__popcll(there) == n) {
    *slots += max(0, end - i0);
    *fixed += n ? outside(i0, end, lo, hi) : 0;
    return;
  }
  for (; there; there &= there - 1) {
    const int i = i0 + 64 * __builtin_ctzll(there), i1 = min(i + 64, to);
    *slots += i1 - i;
    *fixed += outside(i, i1, lo, hi);
  }
}

// The digits of a key from the top: 11, 11 and 10 bits.
struct Digit {
  uint32_t shift, mask, above;      // above: the bits of the digits before it
  __device__ uint32_t of(uint32_t k) const { return (k >> shift) & mask; }
  __device__ bool shares(uint32_t k, uint32_t prefix) const { return ((k ^ prefix) & above) == 0; }
};
__device__ __forceinline__ Digit digit_of(int step) {
  return step == 0 ? Digit{21, 2047, 0} : step == 1 ? Digit{10, 2047, 0xffe00000u} : Digit{0, 1023, 0xfffffc00u};
}

// Adds to hist[d] of every lane with `is`.  Scores repeat (zeros above all), so the digit of the first lane is
// added once for all lanes that have it.
__device__ __forceinline__ void count_digit(uint32_t* hist, bool is, uint32_t d) {
  const uint64_t any = __ballot(is);
  if (any == 0) return;
  const uint32_t first = __builtin_amdgcn_readlane(d, __builtin_ctzll(any));
  const uint64_t same = __ballot(is && d == first);
  if (is && d != first) atomicAdd(&hist[d], 1u);
  if ((threadIdx.x & 63) == __builtin_ctzll(same)) atomicAdd(&hist[first], (uint32_t)__popcll(same));
}

// The digit that holds the want-th largest key, and how many keys lie in larger digits.  Thread t has the
// counts of the two digits that rank 2 t and 2 t + 1 from the top.  With want = 0 it is the top digit, with
// none above.
__device__ __forceinline__ void find_digit(uint32_t c0, uint32_t c1, uint32_t* sums, uint32_t* found, uint32_t want) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int top = kBins - 1 - 2 * tid;
  uint32_t s = c0 + c1;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)s, o);
    if (lane >= o) s += y;
  }
  if (lane == 63) sums[wave] = s;
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

// 2 kept, 1 equal to the threshold, 0 not kept (or no slot: i < 0)
__device__ __forceinline__ int kind_of(int i, uint32_t k, int lo, int hi, uint32_t threshold) {
  if (i < 0) return 0;
  if (i < lo || i >= hi) return 2;
  return k > threshold ? 2 : k == threshold ? 1 : 0;
}

// One workgroup a sequence and kv head; a thread holds kKept keys, kKept kThreads >= n.  512 rows of 4096 to 8192 slots
// take 41 us (0.34 TB/s): bound by the vector instructions of the counting and the listing, 1024 threads a row.
template <int kKept>
__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t sums[kWaves], equals[kWaves], found[2];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = live_slots(a, b);
  int32_t* kept = a.kept + ((int64_t)b * a.kv.heads + h) * a.budget;
  const float* x = a.scores + ((int64_t)b * a.kv.heads + h) * a.slots;
  // slots lo .. hi - 1 compete for the places that the sinks and the recent ones leave; where all fit, none does
  int lo = a.sinks;
  const int hi = n - a.recent;
  if (n <= a.budget) {
    int gone = 0;
    for (int i = tid * kPage; i < n; i += kThreads * kPage) {
      const int32_t p = table_entry(a.kv, b, i / kPage);
      gone |= p < 0 || p >= a.kv.n_pages;
    }
    if (!__syncthreads_or(gone)) {
      if (h == 0 && tid == 0) a.new_len[b] = n;
      for (int i = tid; i < a.budget; i += kThreads) kept[i] = i < n ? i : -1;
      return;
    }
    lo = n;
  }
  // a wavefront has a strip of its own, 64 slots a step
  const int strip = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int from = min(wave * strip, n), to = min(from + strip, n);
  const int32_t entry = entries(a, b, from, kKept, to);
  uint32_t mine[kKept];
#pragma unroll
  for (int j = 0; j < kKept; ++j) {
    const int i = from + 64 * j + lane;
    mine[j] = i < to ? key_of(x[i]) : 0;
  }
  const uint64_t there = pages_there(a, entry);
  // f(slot, key) for the lanes' slots of a strip that are there, all lanes together; a slot past the strip is -1
  auto every = [&](auto f) {
#pragma unroll
    for (int j = 0; j < kKept; ++j)
      if ((there >> j) & 1) {
        const int i = from + 64 * j + lane;
        f(i < to ? i : -1, mine[j]);
      }
  };
  int slots = 0, fixed = 0;
  add_there(there, from, kKept, to, lo, hi, &slots, &fixed);
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  if (lane == 0) {
    sums[wave] = (uint32_t)slots;
    equals[wave] = (uint32_t)fixed;
  }
  __syncthreads();
  slots = fixed = 0;
  for (int w = 0; w < kWaves; ++w) {
    slots += (int)sums[w];
    fixed += (int)equals[w];
  }
  const int m = min(slots, a.budget);
  if (h == 0 && tid == 0) a.new_len[b] = m;
  for (int i = m + tid; i < a.budget; i += kThreads) kept[i] = -1;
  uint32_t want = (uint32_t)(m - fixed);
  uint32_t prefix = 0;
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {
    const Digit d = digit_of(step);
    every([&](int i, uint32_t k) { count_digit(hist, i >= lo && i < hi && d.shares(k, prefix), d.of(k)); });
    __syncthreads();
    const int top = kBins - 1 - 2 * tid;
    const uint32_t c0 = hist[top], c1 = hist[top - 1];
    hist[top] = hist[top - 1] = 0;
    find_digit(c0, c1, sums, found, want);
    prefix |= found[0] << d.shift;
    want -= found[1];
  }
  // kept: keys above prefix, and the first `want` equal to it
  uint32_t na = 0, ne = 0;
  every([&](int i, uint32_t k) {
    const int t = kind_of(i, k, lo, hi, prefix);
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
    const int t = kind_of(i, k, lo, hi, prefix);
    const uint64_t eqs = __ballot(t == 1);
    const bool take = t == 2 || (t == 1 && eq + __popcll(eqs & below) < want);
    const uint64_t takes = __ballot(take);
    if (take) kept[at + __popcll(takes & below)] = i;
    at += __popcll(takes);
    eq += __popcll(eqs);
  });
}

// What the launches of the parts hand on, a row (sequence and kv head) after the other.
struct Parts {
  uint32_t* hist;            // [row][3][parts][kBins]
  uint32_t* state;           // [row][4 + 4 parts]: prefix and want after the first and second digit, then four counts a
                             // part: kept slots before it by the first digit, by the first two; its slots that are there,
                             // those of them that do not compete
  int parts, span;           // slots of a part (whole blocks)
  __device__ uint32_t* hist_of(int64_t row, int step, int part) const { return hist + ((row * 3 + step) * parts + part) * (int64_t)kBins; }
  __device__ uint32_t* state_of(int64_t row) const { return state + row * (4 + 4 * parts); }
};

// The slots that are there, those of them that do not compete, and the latter in parts before this one.
struct There {
  int slots, fixed, fixed_before;
};
__device__ __forceinline__ int wave_sum(int x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ int slots_of(const uint32_t* state, int live) {     // of part `lane` (there are at most 64)
  const int q = threadIdx.x & 63;
  return q < live ? (int)state[4 + 4 * q + 2] : 0;
}
// ... s: slots_of, loaded ahead
__device__ __forceinline__ There there_of(const Parts& p, const uint32_t* state, int s, int part, int live, int n, int lo, int hi) {
  const int q = threadIdx.x & 63;
  if (__all(q >= live || s == min(p.span, n - q * p.span)))
    return There{n, outside(0, n, lo, hi), outside(0, min(part * p.span, n), lo, hi)};
  const int f = q < live ? (int)state[4 + 4 * q + 3] : 0;
  return There{wave_sum(s), wave_sum(f), wave_sum(q < part ? f : 0)};
}

// The digit number `step` from the parts' histograms; returns how many keys of the parts before this one lie in
// larger digits, and (for thread 0 .. all) in *same how many in this digit.  want() is asked for once the histograms are
// on their way.
template <typename Want>
__device__ __forceinline__ uint32_t add_parts(const Parts& p, int64_t row, int step, int part, int live, Want want,
                                              uint32_t* sums, uint32_t* found, uint32_t* shared2, uint32_t* same) {
  const int tid = threadIdx.x, top = kBins - 1 - 2 * tid;
  uint32_t c0 = 0, c1 = 0, b0 = 0, b1 = 0;
  const uint32_t* at = p.hist_of(row, step, 0) + (top - 1);
#pragma unroll 8
  for (int q = 0; q < live; ++q) {
    const uint2 c = *reinterpret_cast<const uint2*>(at + (int64_t)q * kBins);      // (digits top - 1 and top)
    c0 += c.y;
    c1 += c.x;
    if (q < part) {
      b0 += c.y;
      b1 += c.x;
    }
  }
  if (tid < 2) shared2[tid] = 0;
  find_digit(c0, c1, sums, found, want());
  const int digit = (int)found[0];
  uint32_t above = (top > digit ? b0 : 0) + (top - 1 > digit ? b1 : 0);
  for (int o = 32; o; o >>= 1) above += (uint32_t)__shfl_down((int)above, o);
  if ((tid & 63) == 0) atomicAdd(&shared2[0], above);
  if (top == digit) shared2[1] = b0;
  if (top - 1 == digit) shared2[1] = b1;
  __syncthreads();
  *same = shared2[1];
  return shared2[0];
}

// Counts the digit number kDigit of a part's keys; before it, finds the digit before.
template <int kDigit>
__global__ __launch_bounds__(kThreads) void count_kernel(EvictArgs a, Parts p) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t sums[kWaves], found[2], before[2];
  const int part = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = live_slots(a, b), live = (n + p.span - 1) / p.span;
  const bool all = n <= a.budget;                   // every slot that is there is kept: only they are counted
  if ((all && kDigit > 0) || part >= live) return;
  const int64_t row = (int64_t)b * a.kv.heads + h;
  const float* x = a.scores + row * a.slots;
  uint32_t* state = p.state_of(row);
  const int lo = all ? n : a.sinks, hi = n - a.recent;
  const int from = part * p.span, to = min(from + p.span, n);
  float y[kStep];
  int32_t entry;
  auto load = [&](int t) {
    entry = entries(a, b, t + wave * kStep * 64, kStep, to);
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int i = t + (wave * kStep + j) * 64 + lane;
      y[j] = i < to ? x[i] : 0.f;
    }
  };
  load(from);                                       // (on their way while the digit is found)
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  if (kDigit == 0 && tid < 2) before[tid] = 0;
  uint32_t prefix = 0, want = 0;
  if constexpr (kDigit > 0) {
    if constexpr (kDigit > 1) {
      prefix = state[0];
      want = state[1];
    }
    const int mine = kDigit == 1 ? slots_of(state, live) : 0;
    uint32_t same;
    const uint32_t above = add_parts(p, row, kDigit - 1, part, live, [&] {
      if constexpr (kDigit == 1) {
        const There are = there_of(p, state, mine, part, live, n, lo, hi);
        want = (uint32_t)(min(are.slots, a.budget) - are.fixed);
      }
      return want;
    }, sums, found, before, &same);
    prefix |= found[0] << digit_of(kDigit - 1).shift;
    want -= found[1];
    if (tid == 0) {
      uint32_t* mine = state + 4 + 4 * part;
      mine[kDigit - 1] = above + (kDigit > 1 ? mine[0] : 0u);
      if (part == 0) {
        state[2 * (kDigit - 1)] = prefix;
        state[2 * (kDigit - 1) + 1] = want;
      }
    }
  }
  __syncthreads();
  const Digit d = digit_of(kDigit);
  int slots = 0, fixed = 0;
  for (int t = from; t < to; t += kBlock) {
    const int strip = t + wave * kStep * 64;
    if (t != from) load(t);
    const uint64_t there = pages_there(a, entry);
    if (kDigit == 0) add_there(there, strip, kStep, to, lo, hi, &slots, &fixed);
    if (all) continue;
#pragma unroll
    for (int j = 0; j < kStep; ++j)
      if ((there >> j) & 1) {
        const int i = strip + j * 64 + lane;
        const uint32_t k = key_of(y[j]);
        count_digit(hist, i < to && i >= lo && i < hi && d.shares(k, prefix), d.of(k));
      }
  }
  if (kDigit == 0 && lane == 0) {
    atomicAdd(&before[0], (uint32_t)slots);
    atomicAdd(&before[1], (uint32_t)fixed);
  }
  __syncthreads();
  if (kDigit == 0 && tid < 2) state[4 + 4 * part + 2 + tid] = before[tid];
  if (all) return;
  uint32_t* out = p.hist_of(row, kDigit, part);
  for (int i = tid; i < kBins; i += kThreads) out[i] = hist[i];
}

// Finds the last digit and lists a part's kept slots.
__global__ __launch_bounds__(kThreads) void list_kernel(EvictArgs a, Parts p) {
  __shared__ uint32_t sums[kWaves], equals[kWaves], found[2], before[2];
  const int part = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = live_slots(a, b), live = (n + p.span - 1) / p.span;
  const bool all = n <= a.budget;
  const int64_t row = (int64_t)b * a.kv.heads + h;
  int32_t* kept = a.kept + row * a.budget;
  const uint32_t* state = p.state_of(row);
  const int lo = all ? n : a.sinks, hi = n - a.recent;
  const int mine = slots_of(state, live);
  const float* x = a.scores + row * a.slots;
  const int from = part * p.span, to = min(from + p.span, n);
  float y[kStep];
  int32_t entry;
  auto load = [&](int t) {
    entry = entries(a, b, t + wave * kStep * 64, kStep, to);
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int i = t + (wave * kStep + j) * 64 + lane;
      y[j] = i < to ? x[i] : 0.f;
    }
  };
  load(from);                                       // (on their way while the digit is found)
  // places taken before this part: larger keys, the first `want` equal ones, the sinks and the recent ones
  uint32_t at = 0, prefix = 0, want = 0, eq = 0;
  if (!all && part < live) {
    prefix = state[2];
    want = state[3];
    at = add_parts(p, row, 2, part, live, [&] { return want; }, sums, found, before, &eq) + state[4 + 4 * part + 1];
    prefix |= found[0];
    want -= found[1];
    at += min(eq, want);
  }
  const There are = there_of(p, state, mine, part, live, n, lo, hi);
  at += (uint32_t)are.fixed_before;
  const int m = min(are.slots, a.budget);
  const bool as_is = all && m == n;                 // every old slot, in its place
  if (part == 0 && h == 0 && tid == 0) a.new_len[b] = m;
  for (int i = (as_is ? 0 : m) + part * kThreads + tid; i < a.budget; i += p.parts * kThreads) kept[i] = i < m ? i : -1;
  if (as_is || part >= live) return;
  const uint64_t below = (1ull << lane) - 1;
  for (int t = from; t < to; t += kBlock) {
    const int strip = t + wave * kStep * 64;
    if (t != from) load(t);
    const uint64_t there = pages_there(a, entry);
    int kind[kStep];
    uint32_t na = 0, ne = 0;
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int i = strip + j * 64 + lane;
      kind[j] = (there >> j) & 1 ? kind_of(i < to ? i : -1, key_of(y[j]), lo, hi, prefix) : 0;
      na += __popcll(__ballot(kind[j] == 2));
      ne += __popcll(__ballot(kind[j] == 1));
    }
    __syncthreads();                                // the counts of the last block, and those of add_parts, are read
    if (lane == 0) {
      sums[wave] = na;
      equals[wave] = ne;
    }
    __syncthreads();
    uint32_t my_at = at, my_eq = eq;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t taken = sums[w] + (min(eq + equals[w], want) - min(eq, want));
      at += taken;
      eq += equals[w];
      if (w < wave) {
        my_at += taken;
        my_eq += equals[w];
      }
    }
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const uint64_t eqs = __ballot(kind[j] == 1);
      const bool take = kind[j] == 2 || (kind[j] == 1 && my_eq + __popcll(eqs & below) < want);
      const uint64_t takes = __ballot(take);
      if (take) kept[my_at + __popcll(takes & below)] = strip + j * 64 + lane;
      my_at += __popcll(takes);
      my_eq += __popcll(eqs);
    }
  }
}

// A wavefront moves the 64 tokens of a new page and head: a lane looks up one token's old place, then
// D / 16 lanes move a token's codes, 16 bytes each, all loads in flight at once.  2048 of 4096 to 8192 slots of 64
// sequences and 8 heads of 128 channels: 100 us, 2.9 TB/s of the bytes moved; kept tokens lie apart, and what memory
// fetches around their 64 bytes brings it to some 4.
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

namespace {
constexpr int kMaxParts = 64;
int64_t most_slots(const PagedKV& kv, int64_t slots) { return std::min<int64_t>((int64_t)kv.table_pages * kPage, slots); }
int64_t span_of(int64_t most) { return ((most + kMaxParts - 1) / kMaxParts + kBlock - 1) / kBlock * kBlock; }
}  // namespace

size_t evict_workspace_bytes(const PagedKV& kv, int32_t B, int64_t slots) {
  const int64_t most = most_slots(kv, slots);
  if (most <= kHeld * kThreads) return 0;
  const int64_t parts = (most + span_of(most) - 1) / span_of(most);
  return (size_t)B * kv.heads * (3 * parts * kBins + 4 + 4 * parts) * 4;
}

hipError_t launch_cache_evict(const EvictArgs& a, void* workspace, hipStream_t stream) {
  const int64_t most = most_slots(a.kv, a.slots);
  const dim3 g(a.kv.heads, a.B);
  // a strip is whole steps of 64, so a thread holds n / 1024 keys, rounded up
  if (most <= 4 * kThreads) select_kernel<4><<<g, kThreads, 0, stream>>>(a);
  else if (most <= kHeld * kThreads) select_kernel<kHeld><<<g, kThreads, 0, stream>>>(a);
  else {
    Parts p;
    p.span = (int)span_of(most);
    p.parts = (int)((most + p.span - 1) / p.span);
    p.hist = static_cast<uint32_t*>(workspace);
    p.state = p.hist + (int64_t)a.B * a.kv.heads * 3 * p.parts * kBins;
    const dim3 pg(p.parts, a.kv.heads, a.B);
    count_kernel<0><<<pg, kThreads, 0, stream>>>(a, p);
    count_kernel<1><<<pg, kThreads, 0, stream>>>(a, p);
    count_kernel<2><<<pg, kThreads, 0, stream>>>(a, p);
    list_kernel<<<pg, kThreads, 0, stream>>>(a, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.new_slots == 0) return e;
  const dim3 mg((unsigned)((a.new_slots + 4 * kPage - 1) / (4 * kPage)), a.kv.heads, a.B);
  if (a.head_dim == 64) move_kernel<64><<<mg, 256, 0, stream>>>(a);
  else move_kernel<128><<<mg, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace caddtree
