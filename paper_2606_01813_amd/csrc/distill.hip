// The loss, and its gradient, of a drafter that learns from a teacher's top logits.  A row's student is
// q = softmax(l / tau); the teacher lists K tokens with probabilities p_k, and may leave rho to all others:
//     loss = w [ sum_k p_k (log p_k - log q_k) + rho (log rho - log(1 - Q)) ],  Q = sum of q over the listed tokens
//     dloss/dl_v = w / tau [ q_v M - (listed: sum of its p_k; else: rho q_v / (1 - Q)) ],  M = sum_k p_k + rho
// With m the row's largest logit and r the largest of the tokens not listed, e_v = exp((l_v - r) / tau), S the sum of e_v over the
// tokens not listed, f = exp((r - m) / tau) and Z = S f + the listed tokens' exp((l_k - m) / tau): 1 - Q = S f / Z, formed without
// a difference, and its logarithm without f.  A token not listed has the gradient e_v (M f / Z - rho / S) w / tau: one exponential
// and one product, of numbers that are near 1 where the gradient is, however far below the listed tokens the others lie.
//
// A bit for each token says whether it is listed (in LDS): its term is left out of S as the row streams by, and its
// gradient is written by a lane of its own.
//
// Least traffic: each logit read once and each gradient written once.  The gradient needs the row's sums, so a row has to be
// kept or read again; row_kernel does some of both, sums_kernel and grad_kernel do the latter with parts of a few rows.
// Terms are fp32 exponentials of fp32 differences, added in fp64 (one addition a vector of 16 bytes) and joined in fp64.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kMaxK = CADDTREE_MAX_TEACHER;
constexpr int kMine = kMaxK / kWave;              // of the teacher's tokens a lane

// 2^a to a step of fp32, whatever its size: a chain of a few instructions where a row's sums are waited for.
__device__ __forceinline__ double pow2(double a) {
  asm volatile("" : "+v"(a));                     // (as rounded: a product, fused into the difference below, is not near k)
  const double k = rint(a);
  return ldexp((double)__builtin_amdgcn_exp2f((float)(a - k)), (int)fmax(k, -4000.0));
}

// What a row's teacher lists, in LDS.
struct Listed {
  int id[kMaxK];                                  // -1: padding
  double p[kMaxK];
  float l[kMaxK];                                 // the student's logit
  int twice;                                      // a token is listed twice
  float top;                                      // the student's largest logit of them
  double P, A, rho;                               // sum p_k, sum p_k log p_k
};

// How the row's sums enter the gradient.
struct Row {
  float top;                                      // the largest logit, 0 where that is -inf
  float m, k, mc;                                 // terms are exp2((l - m) c - k); m c + k, rounded
  float rest;                                     // gradient of a token not listed / exp2(l c - mc)
  bool far;                                       // ... / exp2((l - m) c - k)
  double Z, mass, scale;                          // M and w / tau
};

// c = log2(e) / tau.  A term is exp2(l c - r), one fused product and difference, where l c stays within kFar: the reference r
// is a product m c as it was rounded, by a half at most, and its distance from m c is made up for in fp64.  Beyond that (masks of
// -1e10 or of the type's lowest value in a whole row, for instance), where the rounding alone would make a term infinite or 0, a
// term is exp2((l - m) c).
constexpr float kFar = 0x1p24f;
constexpr float kRoom = 8.f;                      // a term may reach 2^kRoom before the reference moves

template <int N>
constexpr uint32_t kNone = (1u << N) - 1;         // a lane past the row's end adds none of its vector's
// bits of the N tokens from `at` (a multiple of N) on
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* bits, int at) {
  return reinterpret_cast<const uint8_t*>(bits)[at >> 3] >> (at & 7) & ((1u << N) - 1);
}

// A row's list as it lies in memory.
struct Raw {
  int id[kMaxK];                                  // -1: padding
  float t[kMaxK];                                 // -inf: padding
  float l[kMaxK];
};
// By one wavefront.  The student's logits come from `kept` [K], or where that is NULL from the row, for tokens
// first .. last - 1 (the others may have been overwritten by another workgroup's gradient).
template <typename E>
__device__ void fetch_listed(const DistillArgs& a, int64_t row, const typename E::T* l, const float* kept, int first, int last, Raw& raw) {
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = (int)threadIdx.x % kWave + i * kWave;
    if (k >= a.K) break;
    int id = a.ids[row * a.K + k];
    if ((uint32_t)id >= (uint32_t)a.V) id = -1;
    const float t = a.target[row * a.K + k];
    raw.id[k] = id;
    raw.t[k] = id >= 0 ? t : -INFINITY;
    raw.l[k] = kept ? kept[k] : id >= first && id < last ? (float)l[id] : -INFINITY;
  }
}

// By one wavefront, of a row's list: probabilities, their sums, and the bits of tokens first .. last - 1 (relative to
// first).
__device__ void read_listed(const DistillArgs& a, const Raw& raw, int first, int last, Listed& L, uint32_t* bits) {
  const int lane = (int)threadIdx.x % kWave;
  float top = -INFINITY, most = -INFINITY;
  double z = 0.0, of = 0.0;
  if (!a.tail) {
#pragma unroll 1
    for (int k = lane; k < a.K; k += kWave) top = fmaxf(top, raw.t[k]);
    top = wave_max(top);
    if (top == -INFINITY) top = 0.f;
    double sum = 0.0;
#pragma unroll 1
    for (int k = lane; k < a.K; k += kWave) sum += L.p[k] = exp(((double)raw.t[k] - (double)top) * a.inverse);
    sum = wave_sum(sum);
    z = log(sum);
    of = 1.0 / sum;
  }
  double P = 0.0, A = 0.0;
  bool twice = false;
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave) {
    const int id = raw.id[k], at = id - first;
    const float t = raw.t[k];
    const double logp = a.tail ? (double)t : ((double)t - (double)top) * a.inverse - z;
    const double p = t == -INFINITY ? 0.0 : a.tail ? exp((double)t) : L.p[k] * of;
    P += p;
    if (p != 0.0) A += p * logp;
    if (id >= first && id < last) twice |= (atomicOr(&bits[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u) != 0;
    if (id >= 0) most = fmaxf(most, raw.l[k]);
    L.id[k] = id;
    L.p[k] = p;
    L.l[k] = raw.l[k];
  }
  most = wave_max(most);
  P = wave_sum(P);
  A = wave_sum(A);
  const bool any = __any(twice);
  if (lane == 0) {
    L.twice = any;
    L.top = most;
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

// Of the tokens not listed of a row, or of a part: the largest logit m and the sum of exp((l - m) / tau).
struct Sum {
  float m;
  double s;
};
// A row's sums.  The tokens not listed have exp2((l - rest.m) c - k) as their terms, and f is the size of such a term beside
// the largest logit's.
struct Whole {
  float m;                                        // the largest logit
  double Z;                                       // the sum of exp((l - m) / tau)
  Sum rest;
  int k;
  double f;
  __device__ __forceinline__ double R() const { return rest.s == 0.0 ? 0.0 : rest.s * f; }     // (0: nothing, or less than fp64 has)
};

template <int kN>
__device__ __forceinline__ float top_of(const float (&x)[kN]) {
  float t = x[0];
#pragma unroll
  for (int j = 1; j < kN; ++j) t = fmaxf(t, x[j]);
  return t;
}

// A wavefront's sum as its logits stream by, of those not listed: a listed one may be so far above the others that beside it they
// were nothing.  The reference is the wavefront's and moves seldom: when a logit is kRoom above it.
struct Stream {
  float c, mc, lim, top = -INFINITY;
  double s = 0.0;

  // The first reference is the lowest there is: what is below has no part in s (and where all is, far() says so), what is above
  // moves it up.  So it only rises, and s never grows where it does.
  __device__ __forceinline__ explicit Stream(float c_) : c(c_), mc(-kFar), lim(lowest(c_)) {}
  static __device__ __forceinline__ float lowest(float c) { return (kRoom - kFar) / c; }
  // whether the sum has to be formed again, from differences to its largest logit t
  __device__ __forceinline__ bool far(float t) const { return t > kFar / c || (t > -INFINITY && t <= lowest(c)); }
  template <int kN>
  __device__ __forceinline__ void add(float (&x)[kN], uint32_t on) {
    if (__any(on != 0)) {
#pragma unroll
      for (int j = 0; j < kN; ++j) x[j] = on >> j & 1 ? -INFINITY : x[j];
    }
    const float t = top_of(x);
    top = fmaxf(top, t);
    if (__any(t > lim)) {
      const float m = wave_max(t);
      float r = m * c;
      asm volatile("" : "+v"(r));                 // (as rounded: no part of a fused difference)
      s *= (double)__builtin_amdgcn_exp2f(mc - r);
      mc = r;
      lim = m + kRoom / c;
    }
    float e[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(x[j], c, -mc));
#pragma unroll
    for (int w = 1; w < kN; w <<= 1)
#pragma unroll
      for (int j = 0; j + w < kN; j += 2 * w) e[j] += e[j + w];
    asm volatile("" : "+v"(e[0]));                // (summed here: the terms need no registers after)
    s += (double)e[0];
  }
};

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

// Vectors first .. last - 1 of a row by a workgroup of kThreads, kU loads in flight a lane.  bits: of the first of these
// vectors on; q: what start_stream has asked for.
template <typename E, int kThreads, bool kOnce = false, int kU>
__device__ __forceinline__ void start_stream(Vec<E> (&q)[kU], const typename E::T* l, int first, int last) {
#pragma unroll
  for (int u = 0; u < kU; ++u) q[u] = row_vector<E, kOnce>(l, first + (int)threadIdx.x + u * kThreads, last);
}
template <typename E, int kThreads, bool kOnce = false, int kU>
__device__ __forceinline__ void stream_row(Stream& r, Vec<E> (&q)[kU], const typename E::T* l, int first, int last, const uint32_t* bits) {
  constexpr int N = kN<E>;
  const int lane = (int)threadIdx.x % kWave;
  int at = first + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) * kWave;   // (of the wavefront's first lane)
  const auto add = [&](int u) {
    const int w = at + lane + u * kThreads;
    float x[N];
    __builtin_amdgcn_sched_barrier(0);              // (one vector unpacked at a time: registers)
    q[u].get(x);
    if (at + kU * kThreads < last) q[u] = row_vector<E, kOnce>(l, w + kU * kThreads, last);
    r.add(x, w < last ? bits_at<N>(bits, (w - first) * N) : kNone<N>);
  };
  for (; at + kU * kThreads < last; at += kU * kThreads) {
#pragma unroll
    for (int u = 0; u < kU; ++u) add(u);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u)                      // the last ones, of which there may be fewer
    if (at + u * kThreads < last) add(u);
}

// A wavefront's result, in LDS: its largest logit not listed, and a sum of exp2(l c - r).
struct Partial {
  float top;
  double r, s;
};
// The edge's elements join, and where the terms were too far for the reference they are formed again, from vectors
// first .. last - 1 as stream_row takes them.
template <typename E, int kThreads>
__device__ void put_partial(Stream r, const Edge<E>& edge, const typename E::T* l, int first, int last, const uint32_t* bits,
                            Partial* p) {
  constexpr int N = kN<E>;
  float x[1] = {edge.x};
  r.add(x, edge.on ? 1u : 0u);
  const float top = wave_max(r.top);
  double ref = (double)r.mc;
  if (r.far(top)) {
    r.s = edge.on ? 0.0 : (double)__builtin_amdgcn_exp2f((edge.x - top) * r.c);
    for (int v = first + (int)threadIdx.x; v < last; v += kThreads) {
      const Vec<E> q = Vec<E>::load(l, (uint32_t)v);
      const uint32_t on = bits_at<N>(bits, (v - first) * N);
      float y[N];
      q.get(y);
      for (int j = 0; j < N; ++j) r.s += on >> j & 1 ? 0.0 : (double)__builtin_amdgcn_exp2f((y[j] - top) * r.c);
    }
    ref = (double)top * (double)r.c;
  }
  const double s = wave_sum(r.s);
  if (threadIdx.x % kWave == 0) p[threadIdx.x / kWave] = Partial{top, ref, s};
}
// n partial results joined by one wavefront, in all of its lanes (fixed order).
__device__ __forceinline__ Sum join_partials(const Partial* p, int n, float c) {
  const int w = (int)threadIdx.x % kWave;
  const Partial x = w < n ? p[w] : Partial{-INFINITY, 0.0, 0.0};
  const float m = wave_max(x.top);
  double s = x.s;
  if (m > -INFINITY && s != 0.0) s *= pow2(x.r - (double)m * (double)c);
  return Sum{m, wave_sum(s)};
}

// The listed tokens' part of Z, by one wavefront, in all of its lanes.
__device__ __forceinline__ double listed_sum(const Listed& L, int K, float m, double c) {
  double sum = 0.0;
#pragma unroll 1
  for (int k = (int)threadIdx.x % kWave; k < K; k += kWave) {
    double p;
    if (first_of(L, K, k, p)) sum += L.l[k] == -INFINITY ? 0.0 : pow2(((double)L.l[k] - (double)m) * c);
  }
  return wave_sum(sum);
}

// From the sums of the tokens not listed and of the listed ones, which are relative to the row's largest logit m.
__device__ __forceinline__ Whole whole_of(float m, const Sum& rest, double listed, double c) {
  Whole h;
  h.m = m;
  h.rest = rest;
  h.k = 0;
  h.f = rest.s == 0.0 ? 0.0 : pow2(((double)rest.m - (double)m) * c);
  h.Z = h.R() + listed;
  return h;
}
// From what put_loss kept of them: R, or its logarithm where that is below what a float holds.  The terms are taken relative to
// the power of two next to R, where R is below 1: beside the largest logit they may be nothing.
__device__ __forceinline__ Whole whole_of(const float* stats) {
  Whole h;
  h.m = stats[0];
  h.Z = (double)stats[1];
  const float R = stats[2];
  h.k = 0;
  double s = (double)R;
  if (R < 0.f) {
    h.k = (int)fmaxf(ceilf(R), -2000.f);
    s = pow2((double)R - (double)h.k);
  } else if (R < 1.f && R > 0.f) {
    s = frexp(s, &h.k);
  }
  h.rest = Sum{h.m, s};
  h.f = ldexp(1.0, h.k);
  return h;
}

// The distance of c from c32 grows with that of the terms from m: at k, where they lie, it is made up for.  (A NaN in Z is the
// whole row's.)
__device__ void finish(Row& r, const Whole& h, const Listed& L, float w, const DistillArgs& a) {
  const double k = (double)h.k;
  r.top = h.m == -INFINITY ? 0.f : h.m;
  r.m = h.rest.m == -INFINITY ? 0.f : h.rest.m;
  r.k = (float)h.k;
  const double ref = (double)r.m * (double)a.c32 + k;
  r.mc = (float)ref;
  r.far = !(fabsf(r.mc) <= kFar);
  r.Z = h.Z;
  r.mass = L.P + L.rho;
  r.scale = (double)w * a.inverse;
  const double rest = h.R() == 0.0 ? 0.0 * h.Z : r.scale * (r.mass * h.f / h.Z - (L.rho == 0.0 ? 0.0 : L.rho / h.rest.s));
  r.rest = (float)(rest * pow2((r.far ? 0.0 : (double)r.mc - ref) + k * a.off));
}

// By one wavefront, from the sum of a row's tokens not listed: all its sums, and what its gradient needs.
__device__ __forceinline__ Whole conclude(const DistillArgs& a, const Listed& L, const Sum& rest, float w, Row& r) {
  const float m = fmaxf(rest.m, L.top);
  const Whole h = whole_of(m, rest, listed_sum(L, a.K, m == -INFINITY ? 0.f : m, a.c), a.c);
  if (threadIdx.x % kWave == 0) finish(r, h, L, w, a);
  return h;
}
// ... its loss and stats.
__device__ void put_loss(const DistillArgs& a, int64_t row, const Listed& L, const Whole& h, float w) {
  const int lane = (int)threadIdx.x % kWave;
  const double R = h.R(), logZ = log(h.Z);
  const double from = h.m == -INFINITY ? 0.0 : (double)h.m;
  double x = 0.0;                                 // sum p_k log q_k
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave) {
    if (L.id[k] >= 0 && L.p[k] != 0.0)
      x += L.p[k] * (L.l[k] == -INFINITY ? -INFINITY : ((double)L.l[k] - from) * a.inverse - logZ);
  }
  x = L.A - wave_sum(x);
  if (L.rho > 0.0 && !(R == 0.0)) x += L.rho * (log(L.rho / h.rest.s) - ((double)h.rest.m - from) * a.inverse + logZ);
  if (lane != 0) return;
  a.loss[row] = (float)((double)w * x);
  if (a.stats) {
    a.stats[row * 3] = h.m;
    a.stats[row * 3 + 1] = (float)h.Z;
    a.stats[row * 3 + 2] = (float)(R < 0x1p-126 && R > 0.0 ? log2(h.rest.s) + ((double)h.rest.m - from) * a.c : R);
  }
}

// A vector's gradient into g; the listed tokens' is left to put_listed.  kFarOff: from exp2((l - m) c - k), else m is Row::mc.
template <typename E, bool kFarOff = false>
__device__ __forceinline__ void put_vector(const Vec<E>& q, typename E::T* row, int v, uint32_t on, float m, float rest, float c, float k = 0.f) {
  constexpr int N = kN<E>;
  float x[N];
  q.get(x);
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = __builtin_amdgcn_exp2f(kFarOff ? fmaf(x[j] - m, c, -k) : fmaf(x[j], c, -m)) * rest;
  Vec<E> y;
  y.set(x);
  if (on == 0) {
    y.stream_at(row, (uint32_t)v * 16u);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (!(on >> j & 1)) row[v * N + j] = y.raw(j);
  }
}
template <typename E>
__device__ __forceinline__ void put_edge(const Edge<E>& e, typename E::T* g, const Row& r, float c) {
  if (e.here && !e.on) g[e.at] = (typename E::T)(__builtin_amdgcn_exp2f(r.far ? fmaf(e.x - r.m, c, -r.k) : fmaf(e.x, c, -r.mc)) * r.rest);
}
// Vectors first .. last - 1 of a row, the last first, kU loads in flight a lane.
template <typename E, int kThreads, int kU, bool kFarOff>
__device__ __forceinline__ void put_vectors(const typename E::T* l, typename E::T* g, int first, int last, const uint32_t* bits,
                                            float m, float rest, float c, float k = 0.f) {
  constexpr int kStep = kU * kThreads;
  for (int at = first + (last - first + kStep - 1) / kStep * kStep - kStep; at >= first; at -= kStep) {
    Vec<E> q[kU];
    start_stream<E, kThreads, true>(q, l, at, last);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int v = at + (int)threadIdx.x + u * kThreads;
      if (v < last) put_vector<E, kFarOff>(q[u], g, v, bits_at<kN<E>>(bits, v * kN<E>), m, rest, c, k);
    }
  }
}
// The listed tokens' gradient, of those in first .. last - 1.
template <typename E, int kThreads>
__device__ void put_listed(const DistillArgs& a, typename E::T* g, const Row& r, const Listed& L, int first, int last) {
  for (int k = threadIdx.x; k < a.K; k += kThreads) {
    if (L.id[k] < first || L.id[k] >= last) continue;
    double p;
    if (!first_of(L, a.K, k, p)) continue;
    const double e = L.l[k] == -INFINITY ? 0.0 : pow2(((double)L.l[k] - (double)r.top) * a.c);
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

// A workgroup a row: its loss, and the gradient.  The row's first kKeep vectors a thread stay in registers between the sums
// and the gradient; what is behind them is read again, the last first, while it may still be in a cache.
//
// Bound by memory: 1024 rows of 151936 bf16 (a tenth of weight 0) in 121 to 126 us, 594 MB that have to move at 4.7 to 4.9
// TB/s, where a copy reaches 5.0.  Of 512 threads 0 / 8 / 14 vectors kept: 157 / 129 / 121 us, and 18 were slower than 14; the whole row in
// 1024 threads' registers: 151 when 14 took 136 (one workgroup a compute unit: nothing loads while it joins).
// Streaming stores took 154 to 136, streaming loads of the second pass 133 to 123.
// The loss alone: 2048 such rows in 96 us, 6.2 TB/s of the row's one read; bound by the exponentials' instructions (VALU
// 85% active).  512 threads with 4 / 6 / 8 / 12 loads a lane 94 / 95 / 96 / 99 us, and for 128 rows 17.7 / 16.9 / 16.4 / 16.6;
// 256 threads 97 and 22.
template <typename E, int kThreads, int kKeep, bool kGrad>
__global__ __launch_bounds__(kThreads, 4) void row_kernel(DistillArgs a) {
  constexpr int N = kN<E>, kU = kGrad ? 4 : 8;
  __shared__ Listed L;
  __shared__ Raw raw;
  __shared__ Row r;
  __shared__ Partial part[kThreads / kWave];
  const int b = sequence();
  if (b >= a.B) return;
  const int64_t row = (int64_t)b * a.T + blockIdx.x;
  const int tid = threadIdx.x;
  typename E::T* g = kGrad ? row_of<E>(a.grad, b, blockIdx.x) : nullptr;
  const float w = weight_of(a, row);
  if (w == 0.f) {
    no_weight<E, kThreads>(a, row, g, 0, a.V, true);
    return;
  }
  const typename E::T* l = row_of<E>(a.in, b, blockIdx.x);
  const float c = a.c32;
  const int n = a.V / N, kept = min(n, kKeep * kThreads);          // vectors
  for (int i = tid; i < (a.V + 31) / 32; i += kThreads) s_bits[i] = 0;
  __syncthreads();
  if (tid < kWave) {
    fetch_listed<E>(a, row, l, nullptr, 0, a.V, raw);
    read_listed(a, raw, 0, a.V, L, s_bits);
  }
  Vec<E> q[kKeep > 0 ? kKeep : 1], p[kU];
  if (kKeep > 0 && n > 0) start_stream<E, kThreads, true>(q, l, 0, kept);
  if (kept < n) start_stream<E, kThreads, !kGrad>(p, l, kept, n);
  Edge<E> edge;
  edge.read(l, a.V);
  __syncthreads();
  edge.look(s_bits);
  Stream acc(c);
  int at = tid;                                     // (opaque: no address of a vector is kept until the gradient)
  asm volatile("" : "+v"(at));
  if (kKeep > 0 && n > 0) {
#pragma unroll
    for (int u = 0; u < kKeep; ++u) {
      const int v = u * kThreads + at;
      __builtin_amdgcn_sched_barrier(0);            // (one vector unpacked at a time: registers)
      if (kThreads <= 128 && v - tid % kWave >= n) break;   // (with more threads 1% slower)
      float x[N];
      q[u].get(x);
      acc.add(x, v < n ? bits_at<N>(s_bits, v * N) : kNone<N>);
    }
  }
  if (kept < n) stream_row<E, kThreads, !kGrad>(acc, p, l, kept, n, s_bits + kept * N / 32);
  put_partial<E, kThreads>(acc, edge, l, 0, n, s_bits, part);
  __syncthreads();
  Whole h;
  if (tid < kWave) {
    h = conclude(a, L, join_partials(part, kThreads / kWave, c), w, r);
    if (!kGrad) put_loss(a, row, L, h, w);
  }
  if constexpr (kGrad) {
    __syncthreads();
    const float mc = r.mc, rest = r.rest;
    put_edge<E>(edge, g, r, c);
    if (r.far) {
      put_vectors<E, kThreads, 1, true>(l, g, 0, n, s_bits, r.m, rest, c, r.k);
    } else {
      put_vectors<E, kThreads, kU, false>(l, g, kept, n, s_bits, mc, rest, c);
      asm volatile("" : "+v"(at));
      if constexpr (kKeep > 0) {
#pragma unroll
        for (int u = 0; u < kKeep; ++u) {
          const int v = u * kThreads + at;
          __builtin_amdgcn_sched_barrier(0);
          q[u].forget();
          if (v < n) put_vector<E>(q[u], g, v, bits_at<N>(s_bits, v * N), mc, rest, c);
        }
      }
    }
    put_listed<E, kThreads>(a, g, r, L, 0, a.V);
    if (tid < kWave) put_loss(a, row, L, h, w);
  }
}

// Few rows are cut into parts of `len` tokens (a multiple of 512), a workgroup each: their sums and the listed tokens'
// logits go through the workspace to a second launch.
struct PartSum {
  Sum rest;                                       // of the tokens not listed
  float top;                                      // the largest logit, and from there
  double listed;                                  // ... the sum of the others
};
struct Parts {
  PartSum* sum;                                   // [rows, n]
  float* listed;                                  // [rows, K]
  int n, len;
};
constexpr int kMaxParts = kWave;

// The parts' sums.  Bound by latency: 64 rows of 151936 bf16, 19 MB, in 8 us of which the read at the card's rate is 3; the
// rest is a launch, the list's bits, and two barriers.  Read with the cache's hint, so that the second launch finds the row
// there.  Few wavefronts are sooner under way: 256 / 512 threads 17.6 / 18.0 us in both launches, 16 rows 11.2 / 12.3.
constexpr int kSumThreads = 256;
template <typename E>
__global__ __launch_bounds__(kSumThreads) void sums_kernel(DistillArgs a, Parts ps) {
  __shared__ Partial partial[kSumThreads / kWave];
  __shared__ int s_id[kMaxK];
  __shared__ float s_l[kMaxK];
  __shared__ int s_twice;
  const int t = (int)blockIdx.x / ps.n, part = (int)blockIdx.x % ps.n, tid = threadIdx.x;
  const int64_t row = (int64_t)blockIdx.y * a.T + t;
  if (weight_of(a, row) == 0.f) return;             // (asking for the logits before that gains nothing)
  const int first = part * ps.len, last = min(a.V, first + ps.len);
  const float c = a.c32;
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, t);
  Vec<E> q[6];
  if (first / kN<E> < last / kN<E>) start_stream<E, kSumThreads>(q, l, first / kN<E>, last / kN<E>);
  Edge<E> edge;                                     // (of the row's last part: the others end at a vector's end)
  edge.read(l + first, last - first);
  for (int i = tid; i < (last - first + 31) / 32; i += kSumThreads) s_bits[i] = 0;
  if (tid == 0) s_twice = 0;
  __syncthreads();
  for (int k = tid; k < a.K; k += kSumThreads) {
    int id = a.ids[row * a.K + k];
    if (id < first || id >= last) id = -1;
    s_id[k] = id;
    if (id >= 0) {
      const int at = id - first;
      if (atomicOr(&s_bits[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u) s_twice = 1;
      ps.listed[row * a.K + k] = s_l[k] = (float)l[id];
    }
  }
  __syncthreads();
  edge.look(s_bits);
  Stream acc(c);
  stream_row<E, kSumThreads>(acc, q, l, first / kN<E>, last / kN<E>, s_bits);
  put_partial<E, kSumThreads>(acc, edge, l, first / kN<E>, last / kN<E>, s_bits, partial);
  __syncthreads();
  if (tid >= kWave) return;
  const Sum rest = join_partials(partial, kSumThreads / kWave, c);
  float top = -INFINITY;
  for (int k = tid; k < a.K; k += kWave)
    if (s_id[k] >= 0) top = fmaxf(top, s_l[k]);
  top = fmaxf(wave_max(top), rest.m);
  const double from = top == -INFINITY ? 0.0 : (double)top;
  double listed = 0.0;
  for (int k = tid; k < a.K; k += kWave) {
    bool one = s_id[k] >= 0;
    if (s_twice)
      for (int j = 0; j < k; ++j) one &= s_id[j] != s_id[k];
    if (one && s_l[k] != -INFINITY) listed += pow2(((double)s_l[k] - from) * a.c);
  }
  listed = wave_sum(listed);
  if (tid == 0) ps.sum[row * ps.n + part] = PartSum{rest, top, listed};
}

// A row's sums from its parts', by one wavefront, in all of its lanes.
__device__ __forceinline__ Whole join_parts(const PartSum* p, int n, double c) {
  const int i = (int)threadIdx.x % kWave;
  const PartSum x = i < n ? p[i] : PartSum{{-INFINITY, 0.0}, -INFINITY, 0.0};
  const float m = wave_max(x.rest.m), top = wave_max(x.top);
  double s = x.rest.s, e = x.listed;
  if (m > -INFINITY && s != 0.0) s *= pow2(((double)x.rest.m - (double)m) * c);
  if (top > -INFINITY && e != 0.0) e *= pow2(((double)x.top - (double)top) * c);
  const Sum rest = {m, wave_sum(s)};
  return whole_of(top, rest, wave_sum(e), c);
}

// The gradient of a part of a row.  kStats: from a.stats; else from the parts' sums, and the row's first part writes its
// loss and stats (grad NULL: these alone).
//
// Each workgroup works the list out again, 8 K bytes and K exponentials: that costs less than another launch to do it once.
// One wavefront does, while another joins the parts (one after the other: 64 rows of 151936 19.5 us in both launches, so 18.5).
// From stats a part is what its lanes ask for at once, before the list is gone over.  520 rows of 65537 f16 with K = 128
// (three tenths of weight 0): 29.7 us, 116 MB at 3.9 TB/s; 1024 rows of 151936 bf16: 103 us with 4 loads a lane, 111 with 8.
// Bound by the wait for the list (waits 66% of the wavefronts' cycles), then by memory.  256 / 512 / 1024 threads: from stats
// 103 / 108 / 105 us, behind the sums (a workgroup a compute unit) 20.2 / 17.9 / 18.0.
constexpr int kGradLoads = 4;                     // vectors a lane has in flight while the list is gone over
template <typename E, bool kStats, int kThreads>
__global__ __launch_bounds__(kThreads) void grad_kernel(DistillArgs a, Parts ps) {
  constexpr int N = kN<E>;
  __shared__ Listed L;
  __shared__ Raw raw;
  static_assert(kStats || kThreads >= 2 * kWave, "a wavefront for the list, one for the parts");
  __shared__ Whole s_whole;
  const int t = (int)blockIdx.x / ps.n, part = (int)blockIdx.x % ps.n;
  const int b = sequence();
  if (b >= a.B) return;
  const int64_t row = (int64_t)b * a.T + t;
  const int tid = threadIdx.x, first = part * ps.len, last = min(a.V, first + ps.len);
  typename E::T* g = a.grad.data ? row_of<E>(a.grad, b, t) : nullptr;
  const float w = weight_of(a, row);
  const bool store = !kStats && part == 0;
  if (w == 0.f) {
    no_weight<E, kThreads>(a, row, g, first, last, store);
    return;
  }
  if (g == nullptr && !store) return;
  const typename E::T* l = row_of<E>(a.in, b, t);
  const float c = a.c32;
  const int n = (last - first) / N;
  Vec<E> q[kGradLoads];
  if (g && n > 0) start_stream<E, kThreads, true>(q, l + first, 0, n);
  Edge<E> edge;
  edge.read(l + first, last - first);
  for (int i = tid; i < (last - first + 31) / 32; i += kThreads) s_bits[i] = 0;
  __syncthreads();
  if (tid < kWave) {
    fetch_listed<E>(a, row, l, kStats ? nullptr : ps.listed + row * a.K, first, last, raw);
    read_listed(a, raw, first, last, L, s_bits);
  } else if (!kStats && tid < 2 * kWave) {          // (meanwhile)
    const Whole h = join_parts(ps.sum + row * ps.n, ps.n, a.c);
    if (tid == kWave) s_whole = h;
  }
  Whole h;
  if constexpr (kStats) h = whole_of(a.stats + row * 3);
  __syncthreads();
  if constexpr (!kStats) h = s_whole;
  Row r;                                            // (each for itself)
  finish(r, h, L, w, a);
  if (g) {
    edge.look(s_bits);
    put_edge<E>(edge, g + first, r, c);
    const float mc = r.mc, rest = r.rest;
    if (__builtin_expect(r.far, 0)) {
      put_vectors<E, kThreads, 1, true>(l + first, g + first, 0, n, s_bits, r.m, rest, c, r.k);
    } else {
#pragma unroll
      for (int u = 0; u < kGradLoads; ++u) {
        const int v = u * kThreads + tid;
        __builtin_amdgcn_sched_barrier(0);
        if (v < n) put_vector<E>(q[u], g + first, v, bits_at<N>(s_bits, v * N), mc, rest, c);
      }
      put_vectors<E, kThreads, 4, false>(l + first, g + first, min(n, kGradLoads * kThreads), n, s_bits, mc, rest, c);
    }
    put_listed<E, kThreads>(a, g, r, L, first, last);
  }
  if (store && tid < kWave) put_loss(a, row, L, h, w);
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

// By a row's vectors: as few threads as hold the row, so that many rows are under way, a wavefront alone where that does.
// Measured, us (threads x vectors kept): 65536 rows of 1024 bf16 64 x 4 135, 128 x 4 180; 8192 rows of 8192 64 x 16 57,
// 128 x 14 63, 512 x 0 171; 8192 of 16000 128 x 16 97, 256 x 16 130; 4096 of 32000 256 x 16 96, and when that took 104 512 x 8
// 119, 512 x 14 134; 512 rows of 25000 vectors 512 x 14 64, 1024 x 16 68; 512 rows of 151936 f32 (37984 vectors) 512 x 14
// 148, 1024 x 16 131.  The loss alone: 65536 rows of 1024 64 threads 102, 128 132, 512 496; 16384 of 8192 64 60, 128 63, 512
// 150; 4096 of 32000 64 60, 256 48, 512 58.  (Each with the sums relative to the row's largest logit; relative to the largest of
// the tokens not listed the 65536 rows take 141, their loss 105.)
template <typename E>
hipError_t launch_rows(const DistillArgs& a, hipStream_t stream) {
  const dim3 all = grid_of(a.T, a.B);
  const size_t lds = bit_bytes(a.V);
  const int vectors = a.V / kN<E>;
  if (a.grad.data == nullptr) {
    if (vectors <= 64 * 16) return run(row_kernel<E, 64, 0, false>, all, 64, lds, stream, a);
    if (vectors <= 256 * 16) return run(row_kernel<E, 256, 0, false>, all, 256, lds, stream, a);
    return run(row_kernel<E, 512, 0, false>, all, 512, lds, stream, a);
  }
  if (vectors <= 64 * 4) return run(row_kernel<E, 64, 4, true>, all, 64, lds, stream, a);
  if (vectors <= 64 * 16) return run(row_kernel<E, 64, 16, true>, all, 64, lds, stream, a);
  if (vectors <= 128 * 16) return run(row_kernel<E, 128, 16, true>, all, 128, lds, stream, a);
  if (vectors <= 256 * 16) return run(row_kernel<E, 256, 16, true>, all, 256, lds, stream, a);
  if (vectors <= 1 << 15) return run(row_kernel<E, 512, 14, true>, all, 512, lds, stream, a);
  return run(row_kernel<E, 1024, 16, true>, all, 1024, lds, stream, a);
}

template <typename E>
hipError_t launch_parts(const DistillArgs& a, const Parts& ps, hipStream_t stream) {
  const dim3 g((unsigned)(a.T * ps.n), (unsigned)a.B);
  const hipError_t e = run(sums_kernel<E>, g, kSumThreads, bit_bytes(ps.len), stream, a, ps);
  if (e != hipSuccess) return e;
  return run(grad_kernel<E, false, 512>, g, 512, bit_bytes(ps.len), stream, a, ps);
}

template <typename E>
hipError_t launch(const DistillArgs& a, void* workspace, hipStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.T;
  const int n = workspace ? distill_parts(rows, a.V) : 1;
  if (n <= 1) return launch_rows<E>(a, stream);
  Parts ps;
  ps.len = ((a.V + n - 1) / n + 511) & ~511;
  ps.n = (a.V + ps.len - 1) / ps.len;
  ps.sum = static_cast<PartSum*>(workspace);
  ps.listed = reinterpret_cast<float*>(ps.sum + rows * ps.n);
  return launch_parts<E>(a, ps, stream);
}

template <typename E>
hipError_t launch_grad(const DistillArgs& a, hipStream_t stream) {
  Parts ps = {};
  ps.len = kGradLoads * 256 * kN<E>;
  ps.n = distill_grad_parts(a.V, sizeof(typename E::T));
  const dim3 g = grid_of((int64_t)a.T * ps.n, a.B);
  // (rows shorter than a part: us with 64 / 128 / 256 threads, 65536 rows of 1024 bf16 99 / 104 / 155, 16384 of 4096 56 / 53 / 59;
  // the first 103 with the sums' reference beside R)
  const int vectors = a.V / kN<E>;
  if (vectors <= 64 * 4) return run(grad_kernel<E, true, 64>, g, 64, bit_bytes(ps.len), stream, a, ps);
  if (vectors <= 128 * 4) return run(grad_kernel<E, true, 128>, g, 128, bit_bytes(ps.len), stream, a, ps);
  return run(grad_kernel<E, true, 256>, g, 256, bit_bytes(ps.len), stream, a, ps);
}

}  // namespace

// A workgroup a compute unit where the rows are fewer than that, a part no shorter than what a workgroup asks for at once.
// Parts or whole rows, us, of 151936 bf16: 1 row 8.9 / 24.0, 16 rows 10.4 / 25.3, 64 rows 16.1 / 25.6, 128 rows 25.5 / 26.9
// (their loss alone 17.3 / 16.4, so the rule ends at 64 for both; nothing between was measured); 64 rows of 32000 11.2 / 13.1.  256 or 512 workgroups: 16 rows 11.2 / 12.8, 64 rows
// 17.6 / 18.1, 64 rows of 40000 11.6 / 13.4.
int distill_parts(int64_t rows, int32_t V) {
  if (rows < 1 || rows > 64) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({256 / rows, V / 4096, kMaxParts}));
}
size_t distill_workspace(int64_t rows, int32_t V) {
  const int n = distill_parts(rows, V);
  return n <= 1 ? 0 : (size_t)rows * (n * sizeof(PartSum) + CADDTREE_MAX_TEACHER * sizeof(float));
}

int distill_grad_parts(int32_t V, size_t elem) {
  const int len = kGradLoads * 256 * 16 / (int)elem;
  return (V + len - 1) / len;
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
