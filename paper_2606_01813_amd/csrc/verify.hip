// The target's choice along a built tree: from the root's row on, the largest logit's token (of equals the lowest), then
// the child that carries it, until there is none.  The accepted path is what the target would have written by itself.
//
// Only the rows on the path decide, a handful of a tree's hundreds, and which they are is known one row at a time: a
// workgroup walks a tree and reads a row whenever it gets there.  Where all rows of the call are few, that chain is
// longer than reading them all at once: choose_kernel does so, a workgroup a row, and the walk reads the tokens.

#include <hip/hip_runtime.h>

#include <climits>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

// (x, id) of the larger x, of equals the lower id; nothing yet: (-inf, INT_MAX)
struct Best {
  float x;
  int id;
  __device__ __forceinline__ void take(float y, int i) {
    if (y > x || (y == x && y > -INFINITY && i < id)) {
      x = y;
      id = i;
    }
  }
};

// The token of a row, in every thread: -1 where no logit is above -inf.  s: kWaves places.
template <typename E>
__device__ int choose(const typename E::T* row, int V, Best* s) {
  constexpr int N = kN<E>;
  const int tid = threadIdx.x;
  Best m = {-INFINITY, INT_MAX};
  const int whole = V / N * N;
  for (int at = tid * N; at < whole; at += kThreads * N) {
    float x[N];
    Vec<E>::load(row + at).get(x);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (x[j] > m.x) {                               // (ids only grow: the first of equals stays; NaN is never above)
        m.x = x[j];
        m.id = at + j;
      }
  }
  if (whole + tid < V) m.take((float)row[whole + tid], whole + tid);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m.take(__shfl_xor(m.x, o), __shfl_xor(m.id, o));
  __syncthreads();                                    // (s may still be read, of the row before)
  if (tid % kWave == 0) s[tid / kWave] = m;
  __syncthreads();
  m = s[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m.take(s[w].x, s[w].id);
  return m.id == INT_MAX ? -1 : m.id;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void choose_kernel(VerifyArgs a, int32_t* all) {
  __shared__ Best s[kWaves];
  const int b = (int)blockIdx.y, t = (int)blockIdx.x;
  if (t > min(max(a.count[b], 0), a.T - 1)) return;
  const int id = choose<E>(row_of<E>(a.in, b, t), a.V, s);
  if (threadIdx.x == 0) all[(int64_t)b * a.T + t] = id;
}

// kRead: a row's token comes from its logits, else from a.chosen
template <typename E, bool kRead>
__global__ __launch_bounds__(kThreads) void walk_kernel(VerifyArgs a) {
  __shared__ Best s[kWaves];
  __shared__ int s_child;
  const int b = (int)blockIdx.x, tid = threadIdx.x;
  const int n = min(max(a.count[b], 0), a.T - 1);
  const int32_t* tok = a.token_ids + (int64_t)b * (a.T - 1);
  const int32_t* par = a.parent + (int64_t)b * (a.T - 1);
  if (a.weight)
    for (int i = tid; i < a.T; i += kThreads) a.weight[(int64_t)b * a.T + i] = 0.f;
  int row = 0, steps = 0;
  while (true) {
    int t;
    if constexpr (kRead) t = choose<E>(row_of<E>(a.in, b, row), a.V, s);
    else t = a.chosen[(int64_t)b * a.T + row];
    __syncthreads();                                  // (the weights are cleared, s_child has been read)
    if (tid == 0) {
      a.index[(int64_t)b * a.M + steps] = row;
      a.tokens[(int64_t)b * a.M + steps] = t;
      if (a.weight) a.weight[(int64_t)b * a.T + row] = 1.f;
      s_child = INT_MAX;
    }
    ++steps;
    __syncthreads();
    if (steps >= a.M || t < 0) break;
    // children come after their parent
    for (int i = row + tid; i < n; i += kThreads)
      if (par[i] == row - 1 && tok[i] == t) atomicMin(&s_child, i);
    __syncthreads();
    if (s_child == INT_MAX) break;
    row = s_child + 1;
  }
  if (tid == 0) a.accepted[b] = steps;
  for (int i = steps + tid; i < a.M; i += kThreads) a.index[(int64_t)b * a.M + i] = a.tokens[(int64_t)b * a.M + i] = -1;
}

template <typename E>
void launch(const VerifyArgs& v, int32_t* all, hipStream_t stream) {
  VerifyArgs a = v;
  if (a.in.data != nullptr && all != nullptr) {
    choose_kernel<E><<<dim3((unsigned)a.T, (unsigned)a.B), kThreads, 0, stream>>>(a, all);
    a.chosen = all;
    a.in.data = nullptr;
  }
  if (a.in.data != nullptr) walk_kernel<E, true><<<(unsigned)a.B, kThreads, 0, stream>>>(a);
  else walk_kernel<E, false><<<(unsigned)a.B, kThreads, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, int32_t* all, caddtree_dtype_t dtype, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) launch<BF16>(a, all, stream);
  else if (dtype == CADDTREE_F16) launch<F16>(a, all, stream);
  else launch<F32>(a, all, stream);
  return hipGetLastError();
}

}  // namespace caddtree
