// The loss, and its gradient, of a drafter that learns from a teacher's top logits.  A row's student is
// q = softmax(l / tau); the teacher lists K tokens with probabilities p_k, and may leave rho to all others:
//     loss = w [ sum_k p_k (log p_k - log q_k) + rho (log rho - log(1 - Q)) ],  Q = sum of q over the listed tokens
//     dloss/dl_v = w / tau [ q_v M - (listed: sum of its p_k; else: rho q_v / (1 - Q)) ],  M = sum_k p_k + rho
// With m the row's largest logit, e_v = exp((l_v - m) / tau), R the sum of e_v over the tokens not listed and Z over
// all: q_v = e_v / Z and 1 - Q = R / Z, formed without a difference.  A token not listed has the gradient
// e_v (M / Z - rho / R) w / tau: one exponential and one product.
//
// A bit for each token says whether it is listed (in LDS): its term is left out of R as the row streams by, and its
// gradient is written by a lane of its own.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kMaxK = CADDTREE_MAX_TEACHER;
constexpr int kMine = kMaxK / kWave;              // of the teacher's tokens a lane
constexpr double kLog2e = 0x1.71547652b82fep+0;

// What a row's teacher lists, in LDS.
struct Listed {
  int id[kMaxK];                                  // -1: padding
  double p[kMaxK];
  float l[kMaxK];                                 // the student's logit
  int twice;                                      // a token is listed twice
  double P, A, rho;                               // sum p_k, sum p_k log p_k
};

// How the row's sums enter loss and gradient.
struct Row {
  float m;                                        // the largest logit, 0 where that is -inf
  float rest;                                     // gradient of a token not listed / e_v
  double Z, mass, scale;                          // M and w / tau
};

// bits of the N tokens from `at` (a multiple of N) on
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* bits, int at) {
  return reinterpret_cast<const uint8_t*>(bits)[at >> 3] >> (at & 7) & ((1u << N) - 1);
}

// The listed tokens of a row, by the first wavefront: into L and the bits, those of tokens first .. last - 1 (relative to
// first), with sum p_k and sum p_k log p_k.  Their logits come from `kept` [K], or where that is
// NULL from the row, for tokens first .. last - 1 (the others may have been overwritten by another workgroup's gradient).
template <typename E>
__device__ void read_listed(const DistillArgs& a, int64_t row, const typename E::T* l, const float* kept, int first, int last,
                            Listed& L, uint32_t* bits) {
  const int lane = threadIdx.x;
  int id[kMine];
  float t[kMine], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = lane + i * kWave;
    id[i] = k < a.K ? a.ids[row * a.K + k] : -1;
    if ((uint32_t)id[i] >= (uint32_t)a.V) id[i] = -1;
    t[i] = id[i] >= 0 ? a.target[row * a.K + k] : -INFINITY;
    top = fmaxf(top, t[i]);
  }
  double logp[kMine], p[kMine];
  if (!a.tail) {
    top = wave_max(top);
    if (top == -INFINITY) top = 0.f;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      logp[i] = ((double)t[i] - (double)top) / (double)a.temperature;
      sum += exp(logp[i]);
    }
    const double z = log(wave_sum(sum));
#pragma unroll
    for (int i = 0; i < kMine; ++i) logp[i] = logp[i] == -INFINITY ? -INFINITY : logp[i] - z;
  } else {
#pragma unroll
    for (int i = 0; i < kMine; ++i) logp[i] = (double)t[i];
  }
  double P = 0.0, A = 0.0;
  bool twice = false;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = lane + i * kWave;
    p[i] = exp(logp[i]);
    P += p[i];
    if (p[i] != 0.0) A += p[i] * logp[i];
    const int at = id[i] - first;
    const bool here = id[i] >= first && id[i] < last;
    if (here) twice |= (atomicOr(&bits[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u) != 0;
    if (k < a.K) {
      L.id[k] = id[i];
      L.p[k] = p[i];
      L.l[k] = kept ? kept[k] : here ? (float)l[id[i]] : -INFINITY;
    }
  }
  P = wave_sum(P);
  A = wave_sum(A);
  const bool any = __any(twice);
  if (lane == 0) {
    L.twice = any;
    L.P = P;
    L.A = A;
    L.rho = a.tail && 1.0 - P > 0.0 ? 1.0 - P : 0.0;
  }
}

// whether the k-th is the first of its token, and the sum of the probabilities that its token is listed with
__device__ __forceinline__ bool first_of(const Listed& L, int K, int k, double& p) {
  p = L.p[k];
  if (L.id[k] < 0) return false;
  if (!L.twice) return true;
  p = 0.0;
  bool first = true;
  for (int j = 0; j < K; ++j) {
    if (L.id[j] != L.id[k]) continue;
    first &= j >= k;
    p += L.p[j];
  }
  return first;
}

__device__ __forceinline__ float weight_of(const DistillArgs& a, int64_t row) { return a.weight ? a.weight[row] : 1.f; }

// (m, s): a largest value and a sum of exp((l - m) / tau), joined with another's
__device__ __forceinline__ void join(float& m, double& s, float m2, double s2, float c) {
  const float top = fmaxf(m, m2);
  if (top == -INFINITY) {
    s += s2;                                      // (zeros, or NaN)
    return;
  }
  s = s * (double)__builtin_amdgcn_exp2f((m - top) * c) + s2 * (double)__builtin_amdgcn_exp2f((m2 - top) * c);
  m = top;
}

// A thread's part of a row: its largest logit m and the sum of exp((l - m) / tau) over its tokens not listed.
struct Sum {
  float m = -INFINITY;
  double s = 0.0;
};
template <int kN>
__device__ __forceinline__ float top_of(const float (&x)[kN]) {
  float t = x[0];
#pragma unroll
  for (int j = 1; j < kN; ++j) t = fmaxf(t, x[j]);
  return t;
}
// the sum of a vector's terms, without those of the bits in `on`
template <int kN>
__device__ __forceinline__ float terms(const float (&x)[kN], uint32_t on, float from, float c) {
  float e[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) e[j] = __builtin_amdgcn_exp2f((x[j] - from) * c);
  if (on) {
#pragma unroll
    for (int j = 0; j < kN; ++j) e[j] = on >> j & 1 ? 0.f : e[j];
  }
#pragma unroll
  for (int w = 1; w < kN; w <<= 1)
#pragma unroll
    for (int j = 0; j + w < kN; j += 2 * w) e[j] += e[j + w];
  asm volatile("" : "+v"(e[0]));                  // (summed here: the terms need no registers after)
  return e[0];
}

// Vector v of a row that has n (-inf behind them).
template <typename E>
__device__ __forceinline__ Vec<E> row_vector(const typename E::T* l, int v, int n) {
  Vec<E> q = Vec<E>::neg_inf();
  if (v < n) q = Vec<E>::load(l + v * kN<E>);
  return q;
}

// A row's last elements, fewer than a vector: one in each of the first threads.
template <typename E>
struct Edge {
  int at;
  bool here, on;
  float x;
  __device__ __forceinline__ void read(const typename E::T* l, int V) {
    at = V / kN<E> * kN<E> + (int)threadIdx.x;
    here = at < V;
    x = here ? (float)l[at] : -INFINITY;
  }
  __device__ __forceinline__ void look(const uint32_t* bits) { on = here && (bits[at >> 5] >> (at & 31) & 1u); }
};

// Vectors first .. last - 1 of a row by a workgroup of kThreads, kU loads in flight a lane: the reference moves for a
// wavefront at a time, once for each group of loads.  bits: of the first of these vectors on.
template <typename E, int kThreads, int kU>
__device__ Sum stream_row(const typename E::T* l, int first, int last, float c, const uint32_t* bits) {
  constexpr int N = kN<E>;
  Sum r;
  for (int v0 = first + (int)threadIdx.x; __any(v0 < last); v0 += kU * kThreads) {
    Vec<E> q[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = row_vector<E>(l, v0 + u * kThreads, last);
    float top = r.m;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      __builtin_amdgcn_sched_barrier(0);
      float x[N];
      q[u].get(x);
      top = fmaxf(top, top_of(x));
    }
    if (__any(top > r.m)) {
      top = wave_max(top);
      r.s *= (double)__builtin_amdgcn_exp2f((r.m - top) * c);
      r.m = top;
    }
    const float from = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int v = v0 + u * kThreads;
      __builtin_amdgcn_sched_barrier(0);            // (one vector unpacked at a time: registers)
      q[u].forget();
      float x[N];
      q[u].get(x);
      r.s += (double)terms(x, v < last ? bits_at<N>(bits, (v - first) * N) : 0u, from, c);
    }
  }
  return r;
}

// ... of the row's edge
template <typename E>
__device__ __forceinline__ void take_edge(Sum& r, const Edge<E>& e, float c) {
  if (!e.here) return;
  const float from = e.x == -INFINITY ? 0.f : e.x;
  join(r.m, r.s, e.x, e.on ? 0.0 : (double)__builtin_amdgcn_exp2f(e.x == -INFINITY ? -INFINITY : (e.x - from) * c), c);
}

// The workgroup's sums joined, in all threads (fixed order).
template <int kThreads>
__device__ Sum join_all(Sum r, float c, float* s_m, double* s_s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) join(r.m, r.s, __shfl_xor(r.m, o), __shfl_xor(r.s, o), c);
  if (threadIdx.x % kWave == 0) {
    s_m[threadIdx.x / kWave] = r.m;
    s_s[threadIdx.x / kWave] = r.s;
  }
  __syncthreads();
  r = Sum{s_m[0], s_s[0]};
#pragma unroll
  for (int w = 1; w < kThreads / kWave; ++w) join(r.m, r.s, s_m[w], s_s[w], c);
  return r;
}

// The listed tokens' part of Z, by the first wavefront, in all of its lanes.
__device__ double listed_sum(const Listed& L, int K, float m, double inv_tau) {
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = threadIdx.x + i * kWave;
    double p;
    if (k < K && first_of(L, K, k, p)) sum += L.l[k] == -INFINITY ? 0.0 : exp(((double)L.l[k] - (double)m) * inv_tau);
  }
  return wave_sum(sum);
}

__device__ void finish(Row& r, float m, double Z, double R, const Listed& L, float w, float tau) {
  r.m = m == -INFINITY ? 0.f : m;
  r.Z = Z;
  r.mass = L.P + L.rho;
  r.scale = (double)w / (double)tau;
  r.rest = R == 0.0 ? 0.f : (float)(r.scale * (r.mass / Z - L.rho / R));
}

// Loss and stats of a row, and what its gradient needs, by the first wavefront, from its largest logit and R.
__device__ void conclude(const DistillArgs& a, int64_t row, const Listed& L, Sum sum, float w, Row& r, bool store) {
  const int lane = threadIdx.x;
  const double inv_tau = 1.0 / (double)a.temperature, R = sum.s;
  const float from = sum.m == -INFINITY ? 0.f : sum.m;
  const double Z = R + listed_sum(L, a.K, from, inv_tau), logZ = log(Z);
  double x = 0.0;                                 // sum p_k log q_k
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = lane + i * kWave;
    if (k < a.K && L.id[k] >= 0 && L.p[k] != 0.0)
      x += L.p[k] * (L.l[k] == -INFINITY ? -INFINITY : ((double)L.l[k] - (double)from) * inv_tau - logZ);
  }
  x = L.A - wave_sum(x);
  if (L.rho > 0.0 && !(R == 0.0)) x += L.rho * (log(L.rho) - log(R / Z));
  if (lane == 0) {
    if (store) {
      a.loss[row] = (float)((double)w * x);
      if (a.stats) {
        a.stats[row * 3] = sum.m;
        a.stats[row * 3 + 1] = (float)Z;
        a.stats[row * 3 + 2] = (float)R;
      }
    }
    finish(r, sum.m, Z, R, L, w, a.temperature);
  }
}

// A vector's gradient; the listed tokens' is left to put_listed.
template <typename E>
__device__ __forceinline__ void put_vector(const Vec<E>& q, typename E::T* g, uint32_t on, float m, float rest, float c) {
  constexpr int N = kN<E>;
  float x[N];
  q.get(x);
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = __builtin_amdgcn_exp2f((x[j] - m) * c) * rest;
  Vec<E> v;
  v.set(x);
  if (on == 0) {
    v.store(g);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (!(on >> j & 1)) g[j] = v.raw(j);
  }
}
template <typename E>
__device__ __forceinline__ void put_edge(const Edge<E>& e, typename E::T* g, float m, float rest, float c) {
  if (e.here && !e.on) g[e.at] = (typename E::T)(__builtin_amdgcn_exp2f((e.x - m) * c) * rest);
}
// The listed tokens' gradient, of those in first .. last - 1.
template <typename E, int kThreads>
__device__ void put_listed(const DistillArgs& a, typename E::T* g, const Row& r, const Listed& L, int first, int last) {
  for (int k = threadIdx.x; k < a.K; k += kThreads) {
    if (L.id[k] < first || L.id[k] >= last) continue;
    double p;
    if (!first_of(L, a.K, k, p)) continue;
    const double e = L.l[k] == -INFINITY ? 0.0 : exp(((double)L.l[k] - (double)r.m) / (double)a.temperature);
    g[L.id[k]] = (typename E::T)(float)(r.scale * ((r.Z == 0.0 ? 0.0 : e / r.Z) * r.mass - p));
  }
}

template <typename E, int kThreads>
__device__ void zero_row(typename E::T* g, int first, int last) {
  const Vec<E> zero = {};
  for (int at = first + (int)threadIdx.x * kN<E>; at + kN<E> <= last; at += kThreads * kN<E>) zero.store(g + at);
  const int edge = last - (last - first) % kN<E> + (int)threadIdx.x;
  if (edge < last) g[edge] = (typename E::T)0.f;
}

extern __shared__ uint32_t s_bits[];

// A row of no weight: its gradient's tokens first .. last - 1, loss and stats, are zeros.
template <typename E, int kThreads>
__device__ void no_weight(const DistillArgs& a, int64_t row, typename E::T* g, int first, int last, bool store) {
  if (g) zero_row<E, kThreads>(g, first, last);
  if (store && threadIdx.x == 0) {
    a.loss[row] = 0.f;
    if (a.stats) a.stats[row * 3] = a.stats[row * 3 + 1] = a.stats[row * 3 + 2] = 0.f;
  }
}

// Loss and gradient, a workgroup a row.  The row's first kKeep vectors a thread stay in registers between the sums and the
// gradient; what is behind them is read again.
constexpr int kRowThreads = 1024;
template <typename E, int kKeep>
__global__ __launch_bounds__(kRowThreads) void row_kernel(DistillArgs a) {
  constexpr int N = kN<E>;
  __shared__ Listed L;
  __shared__ Row r;
  __shared__ float s_m[kRowThreads / kWave];
  __shared__ double s_s[kRowThreads / kWave];
  const int64_t row = (int64_t)blockIdx.y * a.T + blockIdx.x;
  const int tid = threadIdx.x;
  typename E::T* g = row_of<E>(a.grad, blockIdx.y, blockIdx.x);
  const float w = weight_of(a, row);
  if (w == 0.f) {
    no_weight<E, kRowThreads>(a, row, g, 0, a.V, true);
    return;
  }
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, blockIdx.x);
  const float c = (float)(kLog2e / (double)a.temperature);
  const int n = a.V / N, kept = min(n, kKeep * kRowThreads);       // vectors
  for (int i = tid; i < (a.V + 31) / 32; i += kRowThreads) s_bits[i] = 0;
  __syncthreads();
  if (tid < kWave) read_listed<E>(a, row, l, nullptr, 0, a.V, L, s_bits);
  Vec<E> q[kKeep];
#pragma unroll
  for (int u = 0; u < kKeep; ++u) q[u] = row_vector<E>(l, u * kRowThreads + tid, n);
  Edge<E> edge;
  edge.read(l, a.V);
  Sum sum;
#pragma unroll
  for (int u = 0; u < kKeep; ++u) {
    __builtin_amdgcn_sched_barrier(0);
    float x[N];
    q[u].get(x);
    sum.m = fmaxf(sum.m, top_of(x));
  }
  sum.m = wave_max(sum.m);
  __syncthreads();                                  // (the bits are set)
  edge.look(s_bits);
  const float from = sum.m == -INFINITY ? 0.f : sum.m;
#pragma unroll
  for (int u = 0; u < kKeep; ++u) {
    const int v = u * kRowThreads + tid;
    __builtin_amdgcn_sched_barrier(0);              // (one vector unpacked at a time: registers)
    q[u].forget();
    float x[N];
    q[u].get(x);
    sum.s += (double)terms(x, v < n ? bits_at<N>(s_bits, v * N) : 0u, from, c);
  }
  if (kept < n) {
    const Sum more = stream_row<E, kRowThreads, 2>(l, kept, n, c, s_bits + kept * N / 32);
    join(sum.m, sum.s, more.m, more.s, c);
  }
  take_edge(sum, edge, c);
  sum = join_all<kRowThreads>(sum, c, s_m, s_s);
  if (tid < kWave) conclude(a, row, L, sum, w, r, true);
  __syncthreads();
  const float m = r.m, rest = r.rest;
#pragma unroll
  for (int u = 0; u < kKeep; ++u) {
    const int v = u * kRowThreads + tid;
    __builtin_amdgcn_sched_barrier(0);
    q[u].forget();
    if (v < n) put_vector<E>(q[u], g + v * N, bits_at<N>(s_bits, v * N), m, rest, c);
  }
  for (int v = kept + tid; v < n; v += kRowThreads)
    put_vector<E>(Vec<E>::load(l + v * N), g + v * N, bits_at<N>(s_bits, v * N), m, rest, c);
  put_edge<E>(edge, g, m, rest, c);
  put_listed<E, kRowThreads>(a, g, r, L, 0, a.V);
}

// The loss alone, a workgroup a row.
constexpr int kLossThreads = 512;
template <typename E>
__global__ __launch_bounds__(kLossThreads) void loss_kernel(DistillArgs a) {
  __shared__ Listed L;
  __shared__ Row r;
  __shared__ float s_m[kLossThreads / kWave];
  __shared__ double s_s[kLossThreads / kWave];
  const int64_t row = (int64_t)blockIdx.y * a.T + blockIdx.x;
  const int tid = threadIdx.x;
  const float w = weight_of(a, row);
  if (w == 0.f) {
    no_weight<E, kLossThreads>(a, row, nullptr, 0, a.V, true);
    return;
  }
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, blockIdx.x);
  const float c = (float)(kLog2e / (double)a.temperature);
  for (int i = tid; i < (a.V + 31) / 32; i += kLossThreads) s_bits[i] = 0;
  __syncthreads();
  if (tid < kWave) read_listed<E>(a, row, l, nullptr, 0, a.V, L, s_bits);
  Edge<E> edge;
  edge.read(l, a.V);
  __syncthreads();
  edge.look(s_bits);
  Sum sum = stream_row<E, kLossThreads, 8>(l, 0, a.V / kN<E>, c, s_bits);
  take_edge(sum, edge, c);
  sum = join_all<kLossThreads>(sum, c, s_m, s_s);
  if (tid < kWave) conclude(a, row, L, sum, w, r, true);
}

// Few rows are cut into parts of `len` tokens (a multiple of 32), a workgroup each: their sums and the listed tokens' logits
// go through the workspace to a second launch.
struct Parts {
  Sum* sum;                                       // [rows, n]
  float* listed;                                  // [rows, K]
  int n, len;
};

constexpr int kSumThreads = 512;
template <typename E>
__global__ __launch_bounds__(kSumThreads) void sums_kernel(DistillArgs a, Parts ps) {
  __shared__ float s_m[kSumThreads / kWave];
  __shared__ double s_s[kSumThreads / kWave];
  const int t = (int)blockIdx.x / ps.n, part = (int)blockIdx.x % ps.n;
  const int64_t row = (int64_t)blockIdx.y * a.T + t;
  if (weight_of(a, row) == 0.f) return;
  const int first = part * ps.len, last = min(a.V, first + ps.len);
  const float c = (float)(kLog2e / (double)a.temperature);
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, t);
  for (int i = threadIdx.x; i < (last - first + 31) / 32; i += kSumThreads) s_bits[i] = 0;
  __syncthreads();
  for (int k = threadIdx.x; k < a.K; k += kSumThreads) {
    const int id = a.ids[row * a.K + k], at = id - first;
    if (id >= first && id < last) {
      atomicOr(&s_bits[at >> 5], 1u << (at & 31));
      ps.listed[row * a.K + k] = (float)l[id];
    }
  }
  __syncthreads();
  Sum sum = stream_row<E, kSumThreads, 8>(l, first / kN<E>, last / kN<E>, c, s_bits);
  Edge<E> edge;                                     // (of the row's last part: the others end at a vector's end)
  edge.read(l + first, last - first);
  edge.look(s_bits);
  take_edge(sum, edge, c);
  sum = join_all<kSumThreads>(sum, c, s_m, s_s);
  if (threadIdx.x == 0) ps.sum[row * ps.n + part] = sum;
}

// The gradient of a part of a row.  kStats: from a.stats; else from the parts' sums, and the row's first part writes its
// loss and stats (grad NULL: these alone).
constexpr int kGradThreads = 256;
template <typename E, bool kStats>
__global__ __launch_bounds__(kGradThreads) void grad_kernel(DistillArgs a, Parts ps) {
  constexpr int N = kN<E>, kU = 4;
  __shared__ Listed L;
  __shared__ Row r;
  const int t = (int)blockIdx.x / ps.n, part = (int)blockIdx.x % ps.n;
  const int64_t row = (int64_t)blockIdx.y * a.T + t;
  const int tid = threadIdx.x, first = part * ps.len, last = min(a.V, first + ps.len);
  typename E::T* g = a.grad.data ? row_of<E>(a.grad, blockIdx.y, t) : nullptr;
  const float w = weight_of(a, row);
  const bool store = !kStats && part == 0;
  if (w == 0.f) {
    no_weight<E, kGradThreads>(a, row, g, first, last, store);
    return;
  }
  if (g == nullptr && !store) return;
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, t);
  const float c = (float)(kLog2e / (double)a.temperature);
  const int b0 = kStats ? first : 0, b1 = kStats ? last : a.V;      // (Z takes the row's listed tokens, each once)
  for (int i = tid; i < (b1 - b0 + 31) / 32; i += kGradThreads) s_bits[i] = 0;
  __syncthreads();
  if (tid < kWave) {
    read_listed<E>(a, row, l, kStats ? nullptr : ps.listed + row * a.K, b0, b1, L, s_bits);
    if constexpr (kStats) {
      if (tid == 0) finish(r, a.stats[row * 3], (double)a.stats[row * 3 + 1], (double)a.stats[row * 3 + 2], L, w, a.temperature);
    } else {
      Sum sum;
      for (int i = 0; i < ps.n; ++i) join(sum.m, sum.s, ps.sum[row * ps.n + i].m, ps.sum[row * ps.n + i].s, c);
      conclude(a, row, L, sum, w, r, store);
    }
  }
  Edge<E> edge;
  edge.read(l + first, last - first);
  __syncthreads();
  if (g == nullptr) return;
  const uint32_t* bits = s_bits + (first - b0) / 32;
  edge.look(bits);
  const float m = r.m, rest = r.rest;
  const int n = (last - first) / N;
  for (int v0 = tid; v0 < n; v0 += kU * kGradThreads) {
    Vec<E> q[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = row_vector<E>(l + first, v0 + u * kGradThreads, n);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int v = v0 + u * kGradThreads;
      if (v < n) put_vector<E>(q[u], g + first + v * N, bits_at<N>(bits, v * N), m, rest, c);
    }
  }
  put_edge<E>(edge, g + first, m, rest, c);
  put_listed<E, kGradThreads>(a, g, r, L, first, last);
}

size_t bit_bytes(int n) { return (size_t)((n + 31) / 32) * 4; }

// A kernel with more LDS than every launch may have has to be told.
template <typename F, typename... A>
hipError_t run(F kernel, dim3 grid, int threads, size_t lds, hipStream_t stream, A... args) {
  if (lds > (40 << 10)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<grid, threads, lds, stream>>>(args...);
  return hipGetLastError();
}

template <typename E>
hipError_t launch_rows(const DistillArgs& a, hipStream_t stream) {
  const dim3 g((unsigned)a.T, (unsigned)a.B);
  const size_t lds = bit_bytes(a.V);
  if (a.grad.data == nullptr) return run(loss_kernel<E>, g, kLossThreads, lds, stream, a);
  const int vectors = (a.V + 1024 * kN<E> - 1) / (1024 * kN<E>);
  if (vectors <= 2) return run(row_kernel<E, 2>, g, 1024, lds, stream, a);
  if (vectors <= 4) return run(row_kernel<E, 4>, g, 1024, lds, stream, a);
  if (vectors <= 8) return run(row_kernel<E, 8>, g, 1024, lds, stream, a);
  if (vectors <= 14) return run(row_kernel<E, 14>, g, 1024, lds, stream, a);
  return run(row_kernel<E, 20>, g, 1024, lds, stream, a);
}

template <typename E>
hipError_t launch_parts(const DistillArgs& a, const Parts& ps, hipStream_t stream) {
  const dim3 g((unsigned)(a.T * ps.n), (unsigned)a.B);
  const hipError_t e = run(sums_kernel<E>, g, kSumThreads, bit_bytes(ps.len), stream, a, ps);
  if (e != hipSuccess) return e;
  return run(grad_kernel<E, false>, g, kGradThreads, bit_bytes(a.V), stream, a, ps);
}

template <typename E>
hipError_t launch(const DistillArgs& a, void* workspace, hipStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.T;
  const int n = workspace ? distill_parts(rows, a.V) : 1;
  if (n <= 1) return launch_rows<E>(a, stream);
  Parts ps;
  ps.len = ((a.V + n - 1) / n + 511) & ~511;
  ps.n = (a.V + ps.len - 1) / ps.len;
  ps.sum = static_cast<Sum*>(workspace);
  ps.listed = reinterpret_cast<float*>(ps.sum + rows * ps.n);
  return launch_parts<E>(a, ps, stream);
}

template <typename E>
hipError_t launch_grad(const DistillArgs& a, hipStream_t stream) {
  Parts ps = {};
  ps.len = 8 * kGradThreads * kN<E>;
  ps.n = (a.V + ps.len - 1) / ps.len;
  return run(grad_kernel<E, true>, dim3((unsigned)(a.T * ps.n), (unsigned)a.B), kGradThreads, bit_bytes(ps.len), stream, a, ps);
}

}  // namespace

int distill_parts(int64_t rows, int32_t V) {
  if (rows < 1 || rows > 128) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(768 / rows, V / 4096));
}
size_t distill_workspace(int64_t rows, int32_t V) {
  const int n = distill_parts(rows, V);
  return n <= 1 ? 0 : (size_t)rows * (n * sizeof(Sum) + CADDTREE_MAX_TEACHER * sizeof(float));
}

hipError_t launch_distill(const DistillArgs& a, void* workspace, caddtree_dtype_t dtype, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) return launch<BF16>(a, workspace, stream);
  if (dtype == CADDTREE_F16) return launch<F16>(a, workspace, stream);
  return launch<F32>(a, workspace, stream);
}
hipError_t launch_distill_grad(const DistillArgs& a, caddtree_dtype_t dtype, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) return launch_grad<BF16>(a, stream);
  if (dtype == CADDTREE_F16) return launch_grad<F16>(a, stream);
  return launch_grad<F32>(a, stream);
}

}  // namespace caddtree
