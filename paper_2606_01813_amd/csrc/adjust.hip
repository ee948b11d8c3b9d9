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
//
// Bound by memory where there are many rows: 1024 rows of 151936 bf16 (histories of up to 2048, 32 biases) in 110 us, 622 MB
// at 5.7 TB/s, 1032 rows of 100003 f32 in a tree with a mask in 118 us.  64 rows with a mask and histories of up to 8192 in
// 17 us: a workgroup has to have gone over the history before its first logit, and VALU is 65% active meanwhile.  In place the
// 1024 rows take 59 us, the 1032 102 and the 64, most of whose tokens are filled one by one, 25.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kChunk = 8192;                      // tokens of a workgroup
// Rows of a workgroup at most: it goes over the history for them all.  1 / 2 / 4 rows: 123 / 110 / 117 us for the 1024 rows,
// 125 / 119 / 147 for the tree's, with histories of 16384 182 / 147 / 161.  256 threads or chunks of 4096 are slower (120 and
// 114 for the 1024 rows).
constexpr int kRows = 2;
constexpr int kMost = 16;                         // ... of a short vocabulary (65536 of 1024 bf16: 2 rows 171 us, 8 55, 16 53, 32 52)
constexpr int kPath = CADDTREE_MAX_L;
constexpr int kNodes = 1024;                      // of a tree, in LDS (further ones are read where they lie)
constexpr int kNear = 512;                        // biases in LDS, likewise
constexpr uint32_t kCount = (1u << 20) - 1;       // a word's count; above it the bias
static_assert(kNear == kThreads, "each thread keeps a bias");
static_assert(CADDTREE_MAX_HISTORY + kPath <= kCount && CADDTREE_MAX_BIAS < 1 << 12, "a word holds both");

struct Lds {
  uint32_t word[kChunk];
  float bias[kNear];
  uint16_t path[kMost][kPath];                    // tokens of a row's path in the chunk, from its first token on
  int paths[kMost];
  int listed;
};
struct Nodes {                                    // of a tree
  uint32_t token[kNodes];
  uint16_t parent[kNodes];                        // + 1
};
extern __shared__ __align__(16) char s_more[];    // a tree's nodes

struct Penalty {
  float repetition, inverse, presence, frequency;
};

// A logit, given its token's word.  The quotient is a product with the inverse: two roundings in place of one, and a tenth
// of the instructions.  (Rounded once, by its remainder: one row 6.4 us instead of 5.6, the 1024 rows 115.5 instead of 110.6.)
__device__ __forceinline__ float adjusted(float x, uint32_t word, const Penalty& p, const Lds& s, const float* bias) {
  const float c = (float)(word & kCount);
  const float y = fmaf(-p.frequency, c, x * (x > 0.f ? p.inverse : p.repetition)) - p.presence;
  x = (word & kCount) != 0 ? y : x;
  const uint32_t place = word >> 20;
  if (place > 0) x += place <= kNear ? s.bias[place - 1] : bias[place - 1];
  return x;
}

// The tokens of the row's path that lie in [from, from + n), relative to from, into path; how many.
__device__ int path_in_chunk(const AdjustArgs& a, const Nodes& s, int b, int row, int from, int n, uint16_t* path) {
  const int64_t base = (int64_t)b * (a.T - 1);
  int node = row - 1, k = 0;
  for (int d = 0; d < kPath && node >= 0; ++d) {
    const int t = (node < kNodes ? (int)s.token[node] : a.token_ids[base + node]) - from;
    const int p = node < kNodes ? (int)s.parent[node] - 1 : a.parent[base + node];
    if ((uint32_t)t < (uint32_t)n) path[k++] = (uint16_t)t;
    node = p < node ? p : -1;
  }
  return k;
}

template <typename E, bool kInPlace>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int shift) {
  __shared__ __align__(16) Lds s;
  __shared__ uint16_t s_list[kInPlace ? kChunk : 1];    // in place: the words that are not 0
  constexpr int N = kN<E>, kStep = kWave * N, kSteps = kChunk / kStep;
  constexpr int kU = kInPlace ? 1 : kRows * kSteps / kWaves;     // loads in flight a lane: all that it has
  // a workgroup takes 2^shift steps of each of its rows
  const int most = min(kRows * kSteps >> shift, kMost);
  constexpr uint32_t kAll = (1u << N) - 1;
  using T = typename E::T;

  const int chunks = (a.V + kChunk - 1) / kChunk;
  const int b = sequence(), first = (int)(blockIdx.x % chunks) * kChunk, last = min(first + kChunk, a.V);
  if (b >= a.B) return;
  const bool tree = a.parent != nullptr;
  const int rows = min(max(a.count ? a.count[b] : a.T - tree, 0), a.T - tree) + tree;   // (rows of the sequence)
  const int row0 = (int)(blockIdx.x / chunks) * most, mine = min(most, rows - row0);
  if (mine <= 0) return;

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // a wavefront takes kStep tokens of a row at a time: step i is i % 2^shift of row i / 2^shift
  const int items = mine << shift;
  const auto token_of = [&](int i) { return first + (i & ((1 << shift) - 1)) * kStep + lane * N; };
  const auto allowed_of = [&](int i, int tok) {         // bit j: token tok + j is allowed
    if (a.allowed == nullptr || tok >= last) return kAll;
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(a.allowed + b * a.allowed_b + (row0 + (i >> shift)) * a.allowed_t);
    return (uint32_t)bytes[tok / 8] >> (tok % 8) & kAll;
  };
  Vec<E> q[kU];
  uint32_t ok[kU];
  const auto ask = [&](int u, int i) {
    if (i >= items) return;
    const int tok = token_of(i);
    ok[u] = allowed_of(i, tok);
    if (!kInPlace && tok + N <= last) {
      const T* src = row_of<E>(a.in, b, row0 + (i >> shift));
      q[u] = Vec<E>::load_once(src, (uint32_t)tok * (uint32_t)sizeof(T));
    }
  };
#pragma unroll
  for (int u = 0; u < kU; ++u) ask(u, wave + u * kWaves);

  // (the first of the biases and of the history are asked for as well, before anything is waited for)
  const int len = a.history ? min(max(a.history_len ? a.history_len[b] : a.H, 0), a.H) : 0;
  const int32_t* history = a.history + (int64_t)b * a.H;
  const int32_t* bias_ids = a.bias_ids + (int64_t)b * a.n_bias;
  const float* bias = a.bias + (int64_t)b * a.n_bias;
  const auto four = [&](int i) { return i + 4 <= a.H ? Vec<F32>::load(reinterpret_cast<const float*>(history) + i) : Vec<F32>{}; };
  Vec<F32> h = a.history ? four(tid * 4) : Vec<F32>{};
  const int bias_id = tid < a.n_bias ? bias_ids[tid] : -1;
  const float bias_value = tid < a.n_bias ? bias[tid] : 0.f;
  const float repetition = a.repetition ? a.repetition[b] : 1.f;
  const Penalty p = {repetition, 1.f / repetition, a.presence ? a.presence[b] : 0.f, a.frequency ? a.frequency[b] : 0.f};
  Nodes& nodes = *reinterpret_cast<Nodes*>(s_more);
  for (int i = tid; i < kStep / 4 << shift; i += kThreads) reinterpret_cast<u32x4*>(s.word)[i] = u32x4{0, 0, 0, 0};
  if (tid == 0) s.listed = 0;
  if (tree)
    for (int i = tid; i < min(row0 + mine - 1, kNodes); i += kThreads) {
      nodes.token[i] = (uint32_t)a.token_ids[(int64_t)b * (a.T - 1) + i];
      const int par = a.parent[(int64_t)b * (a.T - 1) + i];
      nodes.parent[i] = (uint16_t)(par >= 0 && par < i ? par + 1 : 0);
    }
  __syncthreads();
  if (tid < mine) s.paths[tid] = tree ? path_in_chunk(a, nodes, b, row0 + tid, first, last - first, s.path[tid]) : 0;
  const auto found = [&](int w, uint32_t old) {
    if (kInPlace && old == 0) s_list[atomicAdd(&s.listed, 1)] = (uint16_t)w;
  };
  for (int i = tid; i < a.n_bias; i += kThreads) {
    const int t = i == tid ? bias_id : bias_ids[i];
    if (t >= first && t < last) {
      if (i < kNear) s.bias[i] = bias_value;            // (kNear threads: i is this one's)
      found(t - first, atomicMax(&s.word[t - first], (uint32_t)(i + 1) << 20));
    }
  }
  if (a.n_bias > 0) __syncthreads();                    // (the places come before the counts)
  if (len > 0) {
    const auto count = [&](int t) {
      if (t >= first && t < last) found(t - first, atomicAdd(&s.word[t - first], 1u));
    };
    int i = tid * 4;
    while (i + 4 <= len) {
      const Vec<F32> v = h;
      h = four(i + kThreads * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) count((int)v.w[j]);
      i += kThreads * 4;
    }
    for (; i < len; ++i) count(history[i]);             // (fewer than 4, in one thread)
  }
  __syncthreads();

  for (int i0 = wave; i0 < items; i0 += kU * kWaves) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u * kWaves;
      if (i >= items) break;
      const int r = i >> shift, tok = token_of(i);
      T* dst = row_of<E>(a.out, b, row0 + r);
      const uint32_t may = ok[u];
      if constexpr (kInPlace) {
        if (may != kAll) {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (tok + j < last && !(may >> j & 1)) dst[tok + j] = (T)a.fill;
        }
        ask(u, i + kU * kWaves);
      } else {
        Vec<E> v = q[u];
        ask(u, i + kU * kWaves);
        if (tok >= last) continue;
        const bool whole = tok + N <= last;
        uint32_t w[N], any = 0;
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
          const u32x4 four = *reinterpret_cast<const u32x4*>(&s.word[tok - first + 4 * k]);
#pragma unroll
          for (int j = 0; j < 4; ++j) any |= w[4 * k + j] = four[j];
        }
        const int paths = s.paths[r];
        for (int k = 0; k < paths; ++k) {
          const int j0 = first + (int)s.path[r][k] - tok;
          if (j0 >= 0 && j0 < N) {
#pragma unroll
            for (int j = 0; j < N; ++j) w[j] += j0 == j;
            any = 1;
          }
        }
        if (any == 0 && may == kAll && whole) {
          v.stream_at(dst, (uint32_t)tok * (uint32_t)sizeof(T));
          continue;
        }
        float x[N];
        v.get(x);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (!whole) x[j] = tok + j < last ? (float)row_of<E>(a.in, b, row0 + r)[tok + j] : 0.f;
          x[j] = adjusted(x[j], w[j], p, s, bias);
          if (!(may >> j & 1)) x[j] = a.fill;
        }
        if (whole) {
          v.set(x);
          v.stream_at(dst, (uint32_t)tok * (uint32_t)sizeof(T));
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (tok + j < last) dst[tok + j] = (T)x[j];
        }
      }
    }
  }
  if constexpr (kInPlace) {
    // the listed words' tokens and those of the path that are not among them; one not allowed has its value already
    const int listed = s.listed;
    for (int r = wave; r < mine; r += kWaves) {
      T* dst = row_of<E>(a.out, b, row0 + r);
      const uint32_t* allowed = a.allowed ? a.allowed + b * a.allowed_b + (row0 + r) * a.allowed_t : nullptr;
      const int paths = s.paths[r];
      for (int i = lane; i < listed + paths; i += kWave) {
        const int t = first + (i < listed ? s_list[i] : s.path[r][i - listed]);
        if (allowed && !(allowed[t / 32] >> (t % 32) & 1)) continue;
        uint32_t w = s.word[t - first];
        bool again = i >= listed && w != 0;          // of the path, and listed too
        for (int k = 0; k < paths; ++k) {
          const bool same = first + s.path[r][k] == t;
          w += same;
          again |= same && i >= listed && k < i - listed;
        }
        if (!again) dst[t] = (T)adjusted((float)dst[t], w, p, s, bias);
      }
    }
  }
}

template <typename E>
void launch(const AdjustArgs& a, bool in_place, hipStream_t stream) {
  constexpr int kStep = kWave * kN<E>, kSteps = kChunk / kStep;
  int shift = 0;
  while (1 << shift < kSteps && a.V > kStep << shift) ++shift;
  const int most = std::min(kRows * kSteps >> shift, kMost);
  const dim3 g = grid_of((int64_t)((a.V + kChunk - 1) / kChunk) * ((a.T + most - 1) / most), a.B);
  const size_t lds = a.parent != nullptr ? sizeof(Nodes) : 0;
  if (in_place) adjust_kernel<E, true><<<g, kThreads, lds, stream>>>(a, shift);
  else adjust_kernel<E, false><<<g, kThreads, lds, stream>>>(a, shift);
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, caddtree_dtype_t dtype, bool in_place, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) launch<BF16>(a, in_place, stream);
  else if (dtype == CADDTREE_F16) launch<F16>(a, in_place, stream);
  else launch<F32>(a, in_place, stream);
  return hipGetLastError();
}

}  // namespace caddtree
