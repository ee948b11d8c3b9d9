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

#include <cmath>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxK = CADDTREE_MAX_TEACHER;
constexpr int kMine = kMaxK / kWave;              // of the teacher's tokens a lane
constexpr double kLog2e = 0x1.71547652b82fep+0;

// What a row's teacher lists, in LDS.
struct Listed {
  int id[kMaxK];                                  // -1: padding
  double p[kMaxK];
  float l[kMaxK];                                 // the student's logit
  int twice;                                      // a token is listed twice
};

// How the row's sums enter loss and gradient.
struct Row {
  float m;                                        // the largest logit, 0 where that is -inf
  float rest;                                     // gradient of a token not listed / e_v
  double Z, mass, scale;                          // M and w / tau
};

__device__ __forceinline__ void clear_bits(uint32_t* bits, int V) {
  for (int i = threadIdx.x; i < (V + 31) / 32; i += kThreads) bits[i] = 0;
}
// bits of the N tokens from `at` (a multiple of N) on
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* bits, int at) {
  return reinterpret_cast<const uint8_t*>(bits)[at >> 3] >> (at & 7) & ((1u << N) - 1);
}

// The listed tokens of a row, by the first wavefront: into L and the bits; P and A = sum p_k and sum p_k log p_k in all of
// its lanes.
template <typename E>
__device__ void read_listed(const DistillArgs& a, int64_t row, const typename E::T* l, Listed& L, uint32_t* bits, double& P,
                            double& A) {
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
  P = 0.0;
  A = 0.0;
  bool twice = false;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = lane + i * kWave;
    p[i] = exp(logp[i]);
    P += p[i];
    if (p[i] != 0.0) A += p[i] * logp[i];
    if (id[i] >= 0) twice |= (atomicOr(&bits[id[i] >> 5], 1u << (id[i] & 31)) >> (id[i] & 31) & 1u) != 0;
    if (k < a.K) {
      L.id[k] = id[i];
      L.p[k] = p[i];
      L.l[k] = id[i] >= 0 ? (float)l[id[i]] : -INFINITY;
    }
  }
  P = wave_sum(P);
  A = wave_sum(A);
  const bool any = __any(twice);
  if (lane == 0) L.twice = any;
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

// The row's largest logit and the sum R of its tokens not listed, in all threads.
template <typename E>
__device__ void stream_row(const typename E::T* l, int V, float c, const uint32_t* bits, float* s_m, double* s_s, float& m,
                           double& R) {
  constexpr int N = kN<E>;
  const int tid = threadIdx.x;
  float mx = -INFINITY;
  double sum = 0.0;
  for (int at = tid * N; at < V; at += kThreads * N) {
    const int some = min(N, V - at);
    const Packed<E> v = some == N ? Packed<E>::load(l + at) : Packed<E>::load_some(l + at, some);
    const uint32_t on = bits_at<N>(bits, at);
    float top = mx;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < some) top = fmaxf(top, v[j]);
    const float from = top == -INFINITY ? 0.f : top;
    if (top > mx) sum *= (double)__builtin_amdgcn_exp2f((mx - top) * c);
    mx = top;
    float part = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) part += j < some && !(on >> j & 1) ? __builtin_amdgcn_exp2f((v[j] - from) * c) : 0.f;
    sum += (double)part;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) join(mx, sum, __shfl_xor(mx, o), __shfl_xor(sum, o), c);
  if (tid % kWave == 0) {
    s_m[tid / kWave] = mx;
    s_s[tid / kWave] = sum;
  }
  __syncthreads();
  m = s_m[0];
  R = s_s[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) join(m, R, s_m[w], s_s[w], c);
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

__device__ void finish(Row& r, float m, double Z, double R, double P, double rho, float w, float tau) {
  r.m = m == -INFINITY ? 0.f : m;
  r.Z = Z;
  r.mass = P + rho;
  r.scale = (double)w / (double)tau;
  r.rest = R == 0.0 ? 0.f : (float)(r.scale * (r.mass / Z - rho / R));
}

template <typename E>
__device__ void write_grad(const DistillArgs& a, const typename E::T* l, typename E::T* g, const Row& r, const Listed& L,
                           const uint32_t* bits) {
  constexpr int N = kN<E>;
  const float c = (float)(kLog2e / (double)a.temperature), m = r.m, rest = r.rest;
  for (int at = threadIdx.x * N; at < a.V; at += kThreads * N) {
    const int some = min(N, a.V - at);
    Packed<E> v = some == N ? Packed<E>::load(l + at) : Packed<E>::load_some(l + at, some);
    const uint32_t on = bits_at<N>(bits, at);
#pragma unroll
    for (int j = 0; j < N; ++j) v.set(j, __builtin_amdgcn_exp2f((v[j] - m) * c) * rest);
    if (some == N && on == 0) {
      v.store(g + at);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < some && !(on >> j & 1)) g[at + j] = v.v[j];
    }
  }
  for (int k = threadIdx.x; k < a.K; k += kThreads) {
    double p;
    if (!first_of(L, a.K, k, p)) continue;
    const double e = L.l[k] == -INFINITY ? 0.0 : exp(((double)L.l[k] - (double)m) / (double)a.temperature);
    g[L.id[k]] = (typename E::T)(float)(r.scale * ((r.Z == 0.0 ? 0.0 : e / r.Z) * r.mass - p));
  }
}

template <typename E>
__device__ void zero_row(typename E::T* g, int V) {
  constexpr int N = kN<E>;
  const Packed<E> zero = {};
  for (int at = threadIdx.x * N; at < V; at += kThreads * N) {
    if (V - at >= N) zero.store(g + at);
    else zero.store_some(g + at, V - at);
  }
}

extern __shared__ uint32_t s_bits[];

// kStats: the sums come from a.stats, and the gradient alone is written
template <typename E, bool kStats>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  __shared__ Listed L;
  __shared__ Row r;
  __shared__ float s_m[kWaves];
  __shared__ double s_s[kWaves];
  const int64_t row = (int64_t)blockIdx.y * a.T + blockIdx.x;
  const int tid = threadIdx.x;
  typename E::T* g = a.grad.data ? row_of<E>(a.grad, blockIdx.y, blockIdx.x) : nullptr;
  const float w = weight_of(a, row);
  if (w == 0.f) {
    if (g) zero_row<E>(g, a.V);
    if (!kStats && tid == 0) {
      a.loss[row] = 0.f;
      if (a.stats) a.stats[row * 3] = a.stats[row * 3 + 1] = a.stats[row * 3 + 2] = 0.f;
    }
    return;
  }
  const typename E::T* l = row_of<E>(a.in, blockIdx.y, blockIdx.x);
  const float c = (float)(kLog2e / (double)a.temperature);
  clear_bits(s_bits, a.V);
  __syncthreads();
  double P = 0.0, A = 0.0;
  if (tid < kWave) read_listed<E>(a, row, l, L, s_bits, P, A);
  __syncthreads();
  const double rho = a.tail && 1.0 - P > 0.0 ? 1.0 - P : 0.0;
  if constexpr (kStats) {
    if (tid == 0) finish(r, a.stats[row * 3], (double)a.stats[row * 3 + 1], (double)a.stats[row * 3 + 2], P, rho, w, a.temperature);
  } else {
    float m;
    double R;
    stream_row<E>(l, a.V, c, s_bits, s_m, s_s, m, R);
    if (tid < kWave) {
      const double inv_tau = 1.0 / (double)a.temperature;
      const float from = m == -INFINITY ? 0.f : m;
      const double Z = R + listed_sum(L, a.K, from, inv_tau), logZ = log(Z);
      double x = 0.0;                             // sum p_k log q_k
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int k = tid + i * kWave;
        if (k < a.K && L.id[k] >= 0 && L.p[k] != 0.0)
          x += L.p[k] * (L.l[k] == -INFINITY ? -INFINITY : ((double)L.l[k] - (double)from) * inv_tau - logZ);
      }
      x = A - wave_sum(x);
      if (rho > 0.0 && !(R == 0.0)) x += rho * (log(rho) - log(R / Z));
      if (tid == 0) {
        a.loss[row] = (float)((double)w * x);
        if (a.stats) {
          a.stats[row * 3] = m;
          a.stats[row * 3 + 1] = (float)Z;
          a.stats[row * 3 + 2] = (float)R;
        }
        finish(r, m, Z, R, P, rho, w, a.temperature);
      }
    }
  }
  if (g == nullptr) return;
  __syncthreads();
  write_grad<E>(a, l, g, r, L, s_bits);
}

template <typename E, bool kStats>
void launch(const DistillArgs& a, hipStream_t stream) {
  const size_t bytes = (size_t)((a.V + 31) / 32) * 4;
  distill_kernel<E, kStats><<<dim3((unsigned)a.T, (unsigned)a.B), kThreads, bytes, stream>>>(a);
}
template <bool kStats>
hipError_t launch_type(const DistillArgs& a, caddtree_dtype_t dtype, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) launch<BF16, kStats>(a, stream);
  else if (dtype == CADDTREE_F16) launch<F16, kStats>(a, stream);
  else launch<F32, kStats>(a, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, caddtree_dtype_t dtype, hipStream_t stream) {
  return launch_type<false>(a, dtype, stream);
}
hipError_t launch_distill_grad(const DistillArgs& a, caddtree_dtype_t dtype, hipStream_t stream) {
  return launch_type<true>(a, dtype, stream);
}

}  // namespace caddtree
