// Penalties for repeated tokens, biases and a grammar's mask on rows of logits:
//     c > 0:  x = x > 0 ? x / repetition : x repetition;  x = x - frequency c - presence
//     x += bias of v;  x = fill (-inf, or a finite value) where v is not allowed
// with c the number of times that token v stands in the sequence's history and, in a tree, on the row's path.
//
// A workgroup takes kChunk tokens of the vocabulary for a group of a sequence's rows.  It goes over the sequence's
// biases and history once and keeps, in LDS, a word for each of its tokens: how often it occurred (20 bits) and which
// bias it has (12 bits: its place in the list + 1, the largest of a token listed twice).  Integer sums and maxima, so
// their order does not matter.  A row's path adds to that: at most 32 tokens, kept apart, of which few lie in a chunk.
//
// Out of place a wavefront streams a row's part of the chunk, 16 bytes a lane.  In place it touches only what
// changes: the tokens with a word (listed as they are found), those on the row's path, and those not allowed.

#include <hip/hip_runtime.h>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kChunk = 8192;                      // tokens of a workgroup
constexpr int kRows = 16;                         // rows of a workgroup at most
constexpr int kPath = CADDTREE_MAX_L;
constexpr uint32_t kCount = (1u << 20) - 1;       // a word's count; above it the bias
static_assert(CADDTREE_MAX_HISTORY + kPath <= kCount && CADDTREE_MAX_BIAS < 1 << 12, "a word holds both");

struct Penalty {
  float repetition, presence, frequency;
};

// A logit, given how often its token occurred and its bias's place in the sequence's list + 1 (0: none).
__device__ __forceinline__ float adjusted(float x, int c, uint32_t place, const Penalty& p, const float* bias) {
  if (c > 0) {
    x = x > 0.f ? x / p.repetition : x * p.repetition;
    x = fmaf(-p.frequency, (float)c, x) - p.presence;
  }
  if (place > 0) x += bias[place - 1];
  return x;
}

// The tokens of the row's path that lie in [first, first + n), relative to first, into path; how many.
__device__ int path_in_chunk(const AdjustArgs& a, int b, int row, int first, int n, uint16_t* path) {
  const int64_t base = (int64_t)b * (a.T - 1);
  int node = row - 1, k = 0;
  for (int d = 0; d < kPath && node >= 0; ++d) {
    const int t = a.token_ids[base + node] - first;
    const int p = a.parent[base + node];
    if ((uint32_t)t < (uint32_t)n) path[k++] = (uint16_t)t;
    node = p < node ? p : -1;
  }
  return k;
}

template <typename E, bool kInPlace>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a) {
  __shared__ uint32_t s_word[kChunk];
  __shared__ uint16_t s_list[kInPlace ? kChunk : 1];    // in place: the tokens that have a word
  __shared__ uint16_t s_path[kRows][kPath];
  __shared__ int s_paths[kRows];
  __shared__ int s_listed;
  constexpr int N = kN<E>;
  using T = typename E::T;

  const int b = (int)blockIdx.z, first = (int)blockIdx.x * kChunk, n = min(kChunk, a.V - first);
  const bool tree = a.parent != nullptr;
  const int rows = min(max(a.count ? a.count[b] : a.T - tree, 0), a.T - tree) + tree;   // (rows of the sequence)
  const int row0 = (int)blockIdx.y * kRows, mine = min(kRows, rows - row0);
  if (mine <= 0) return;

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const Penalty p = {a.repetition ? a.repetition[b] : 1.f, a.presence ? a.presence[b] : 0.f, a.frequency ? a.frequency[b] : 0.f};
  const float* bias = a.bias + (int64_t)b * a.n_bias;
  for (int i = tid; i < kChunk; i += kThreads) s_word[i] = 0;
  if (tid == 0) s_listed = 0;
  if (tid < mine) s_paths[tid] = tree ? path_in_chunk(a, b, row0 + tid, first, n, s_path[tid]) : 0;
  __syncthreads();
  for (int i = tid; i < a.n_bias; i += kThreads) {
    const int t = a.bias_ids[(int64_t)b * a.n_bias + i] - first;
    if ((uint32_t)t < (uint32_t)n) {
      const uint32_t old = atomicMax(&s_word[t], (uint32_t)(i + 1) << 20);
      if (kInPlace && old == 0) s_list[atomicAdd(&s_listed, 1)] = (uint16_t)t;
    }
  }
  __syncthreads();
  if (a.history != nullptr) {
    const int len = min(max(a.history_len ? a.history_len[b] : a.H, 0), a.H);
    const int32_t* h = a.history + (int64_t)b * a.H;
    for (int i = tid; i < len; i += kThreads) {
      const int t = h[i] - first;
      if ((uint32_t)t < (uint32_t)n) {
        const uint32_t old = atomicAdd(&s_word[t], 1u);
        if (kInPlace && old == 0) s_list[atomicAdd(&s_listed, 1)] = (uint16_t)t;
      }
    }
  }
  __syncthreads();

  // a wavefront takes kStep tokens of a row at a time
  constexpr int kStep = kWave * N;
  const int steps = (n + kStep - 1) / kStep;
  for (int i = wave; i < mine * steps; i += kWaves) {
    const int r = i / steps, at = (i % steps) * kStep + lane * N;
    const T* src = row_of<E>(a.in, b, row0 + r) + first;
    T* dst = row_of<E>(a.out, b, row0 + r) + first;
    const int some = min(N, n - at);
    if (some <= 0) continue;
    uint32_t ok = 0xffffffffu;                      // bit j: token at + j is allowed
    if (a.allowed != nullptr) {
      const uint8_t* bytes = reinterpret_cast<const uint8_t*>(a.allowed + b * a.allowed_b + (row0 + r) * a.allowed_t);
      ok = bytes[(first + at) / 8] >> ((first + at) % 8);
    }
    if constexpr (kInPlace) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < some && !(ok >> j & 1)) dst[j + at] = (T)a.fill;
    } else {
      const int paths = s_paths[r];
      float x[N];
      Vec<E> v;
      if (some == N) {
        v = Vec<E>::load(src + at);
        v.get(x);
      }
      bool change = false;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (some < N) x[j] = j < some ? (float)src[at + j] : 0.f;
        const uint32_t w = s_word[min(at + j, kChunk - 1)];
        int c = (int)(w & kCount);
        for (int k = 0; k < paths; ++k) c += s_path[r][k] == at + j;
        if (c > 0 || w >> 20) x[j] = adjusted(x[j], c, w >> 20, p, bias);
        if (!(ok >> j & 1)) x[j] = a.fill;
        change |= c > 0 || w >> 20 || !(ok >> j & 1);
      }
      if (some == N) {
        if (change) v.set(x);
        v.store(dst + at);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < some) dst[at + j] = (T)x[j];
      }
    }
  }
  if constexpr (kInPlace) {
    // the listed tokens and those of the path that are not among them; one not allowed has its value already
    const int listed = s_listed;
    for (int r = wave; r < mine; r += kWaves) {
      T* dst = row_of<E>(a.out, b, row0 + r) + first;
      const uint32_t* allowed = a.allowed ? a.allowed + b * a.allowed_b + (row0 + r) * a.allowed_t : nullptr;
      const int paths = s_paths[r];
      for (int i = lane; i < listed + paths; i += kWave) {
        const int t = i < listed ? s_list[i] : s_path[r][i - listed];
        if (allowed && !(allowed[(first + t) / 32] >> ((first + t) % 32) & 1)) continue;
        const uint32_t w = s_word[t];
        int c = (int)(w & kCount);
        bool again = i >= listed && w != 0;          // of the path, and listed too
        for (int k = 0; k < paths; ++k) {
          const bool same = s_path[r][k] == t;
          c += same;
          again |= same && i >= listed && k < i - listed;
        }
        if (!again) dst[t] = (T)adjusted((float)dst[t], c, w >> 20, p, bias);
      }
    }
  }
}

template <typename E>
void launch(const AdjustArgs& a, bool in_place, hipStream_t stream) {
  const dim3 g((unsigned)((a.V + kChunk - 1) / kChunk), (unsigned)((a.T + kRows - 1) / kRows), (unsigned)a.B);
  if (in_place) adjust_kernel<E, true><<<g, kThreads, 0, stream>>>(a);
  else adjust_kernel<E, false><<<g, kThreads, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, caddtree_dtype_t dtype, bool in_place, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) launch<BF16>(a, in_place, stream);
  else if (dtype == CADDTREE_F16) launch<F16>(a, in_place, stream);
  else launch<F32>(a, in_place, stream);
  return hipGetLastError();
}

}  // namespace caddtree
