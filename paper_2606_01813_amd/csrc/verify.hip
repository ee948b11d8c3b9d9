// The target's choice along a built tree: from the root's row on, the largest logit's token (of equals the lowest), then
// the child that carries it, until there is none.  The accepted path is what the target would have written by itself.
//
// Only the rows on the path decide, a handful of a tree's hundreds, and which they are is known one row at a time: a
// workgroup walks a tree and reads a row whenever it gets there.  Where all rows of the call are few, that chain is
// longer than reading them all at once: choose_kernel does so, a part of a row a workgroup, and the walk joins the parts.
//
// 32 trees of up to 256 nodes, 151936 bf16 logits a row, take 55 us: the longest path's rows one after the other, each at what
// a compute unit reads of its 304 KB.  One tree of 64 nodes: 12 us, all rows at once in 6.5 and the walk over the parts in 6.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kWalkThreads = 1024;
constexpr int kChooseThreads = 256;
constexpr int kNodes = 2048;                      // of a tree, in LDS (further ones are read where they lie)

// (x, id) of the larger x, of equals the lower id; nothing yet: (-inf, INT_MAX)
struct Best {
  float x;
  int id;
  __device__ __forceinline__ void take(float y, int i) {
    if (y > x || (y == x && i < id)) {
      x = y;
      id = i;
    }
  }
  // over a wavefront, in all of its lanes
  __device__ __forceinline__ void join() {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) take(__shfl_xor(x, o), __shfl_xor(id, o));
  }
  __device__ __forceinline__ int token() const { return x > -INFINITY ? id : -1; }
};

// The best of a row's tokens first .. last - 1 (first a multiple of 8) by a workgroup, kU loads in flight a lane; in each
// wavefront its own.  A lane keeps the vector with the largest logit, the first of equals; which of its elements that is
// is looked for once, at the end.
// The walk with 5 / 10 / 20 loads a lane: 55.2 / 56.4 / 92 us (20 leave room for too few wavefronts).
template <typename E, int kThreads, int kU>
__device__ Best best_of(const typename E::T* row, int first, int last) {
  constexpr int N = kN<E>;
  const int n = last / N, lane = (int)(threadIdx.x % kWave);
  const int edge = n * N + (int)threadIdx.x;
  const float rest = edge < last && threadIdx.x < N ? (float)row[edge] : -INFINITY;
  int v = first / N + (int)threadIdx.x;
  Vec<E> q[kU], best = Vec<E>::neg_inf();
  if (v - lane < n) {
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = row_vector<E>(row, v + u * kThreads, n);
  }
  float top = -INFINITY;
  int at = 0;
  for (; v - lane < n; v += kU * kThreads) {          // (past the end a lane sees the last vector again)
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float x[N];
      __builtin_amdgcn_sched_barrier(0);              // (one vector unpacked at a time: registers)
      q[u].get(x);
      float t = x[0];
#pragma unroll
      for (int j = 1; j < N; ++j) t = fmaxf(t, x[j]);
      const bool up = t > top;                        // (vectors only grow: the first of equals stays; NaN is never above)
      top = up ? t : top;
      at = up ? min(v + u * kThreads, n - 1) : at;
#pragma unroll
      for (int j = 0; j < 4; ++j) best.w[j] = up ? q[u].w[j] : best.w[j];
      q[u] = row_vector<E>(row, v + (u + kU) * kThreads, n);
    }
  }
  float x[N];
  best.get(x);
  int place = N - 1;
#pragma unroll
  for (int j = N - 2; j >= 0; --j) place = x[j] == top ? j : place;
  Best m = {top, top > -INFINITY ? at * N + place : INT_MAX};
  if (rest > -INFINITY) m.take(rest, edge);
  m.join();
  return m;
}

// Part blockIdx.x of row blockIdx.y of tree blockIdx.z: parts [B, T, n], of len tokens (a multiple of 8)
template <typename E>
__global__ __launch_bounds__(kChooseThreads) void choose_kernel(VerifyArgs a, Best* parts, int len) {
  __shared__ Best s[kChooseThreads / kWave];
  const int b = (int)blockIdx.z, t = (int)blockIdx.y, first = (int)blockIdx.x * len;
  if (t > min(max(a.count[b], 0), a.T - 1)) return;
  const Best m = best_of<E, kChooseThreads, 4>(row_of<E>(a.in, b, t), first, min(first + len, a.V));
  if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = m;
  __syncthreads();
  if (threadIdx.x != 0) return;
  Best all = s[0];
#pragma unroll
  for (int w = 1; w < kChooseThreads / kWave; ++w) all.take(s[w].x, s[w].id);
  parts[((int64_t)b * a.T + t) * gridDim.x + blockIdx.x] = all;
}

enum Source { kRead, kParts, kChosen };               // where a row's token comes from: its logits, their parts, the caller
template <typename E, Source kFrom, int kThreads>
__global__ __launch_bounds__(kThreads) void walk_kernel(VerifyArgs a, const Best* parts, int n_parts) {
  __shared__ Best s[kThreads / kWave];
  __shared__ uint32_t s_token[kNodes];
  __shared__ uint16_t s_parent[kNodes];               // + 1
  __shared__ int s_child;
  const int b = (int)blockIdx.x, tid = threadIdx.x;
  const int n = min(max(a.count[b], 0), a.T - 1);
  const int32_t* tok = a.token_ids + (int64_t)b * (a.T - 1);
  const int32_t* par = a.parent + (int64_t)b * (a.T - 1);
  for (int i = tid; i < min(n, kNodes); i += kThreads) {
    const int p = par[i];
    s_token[i] = (uint32_t)tok[i];
    s_parent[i] = (uint16_t)(p >= -1 && p < i ? p + 1 : 0xffff);     // (no child of any row: children come after their parent)
  }
  if (a.weight)
    for (int i = tid; i < a.T; i += kThreads) a.weight[(int64_t)b * a.T + i] = 0.f;
  int row = 0, steps = 0;
  while (true) {
    Best m;
    if constexpr (kFrom == kRead) {
      m = best_of<E, kThreads, 5>(row_of<E>(a.in, b, row), 0, a.V);
      if (tid % kWave == 0) s[tid / kWave] = m;
    } else if constexpr (kFrom == kParts) {
      const int i = tid % kWave;
      m = i < n_parts ? parts[((int64_t)b * a.T + row) * n_parts + i] : Best{-INFINITY, INT_MAX};
      m.join();
    }
    if (tid == 0) s_child = INT_MAX;
    __syncthreads();                                  // (the weights are cleared too, and the nodes are there)
    int t;
    if constexpr (kFrom == kRead) {
      m = tid % kWave < kThreads / kWave ? s[tid % kWave] : Best{-INFINITY, INT_MAX};
      m.join();
    }
    if constexpr (kFrom == kChosen) t = a.chosen[(int64_t)b * a.T + row];
    else t = m.token();
    if (tid == 0) {
      a.index[(int64_t)b * a.M + steps] = row;
      a.tokens[(int64_t)b * a.M + steps] = t;
      if (a.weight) a.weight[(int64_t)b * a.T + row] = 1.f;
    }
    ++steps;
    if (steps >= a.M || t < 0) break;
    for (int i = row + tid; i < n; i += kThreads)
      if (i < kNodes ? s_parent[i] == row && (int)s_token[i] == t : par[i] == row - 1 && tok[i] == t) atomicMin(&s_child, i);
    __syncthreads();
    const int child = s_child;
    if (child == INT_MAX) break;
    row = child + 1;
    __syncthreads();                                  // (s and s_child have been read)
  }
  if (tid == 0) a.accepted[b] = steps;
  for (int i = steps + tid; i < a.M; i += kThreads) a.index[(int64_t)b * a.M + i] = a.tokens[(int64_t)b * a.M + i] = -1;
}

template <typename E>
void launch(const VerifyArgs& a, void* workspace, size_t elem, hipStream_t stream) {
  if (a.in.data == nullptr) {
    walk_kernel<E, kChosen, 256><<<(unsigned)a.B, 256, 0, stream>>>(a, nullptr, 0);
    return;
  }
  const int n = workspace ? verify_parts(a.B, a.T, a.V, elem) : 0;
  if (n == 0) {
    walk_kernel<E, kRead, kWalkThreads><<<(unsigned)a.B, kWalkThreads, 0, stream>>>(a, nullptr, 0);
    return;
  }
  const int len = ((a.V + n - 1) / n + 7) & ~7;
  const int parts = (a.V + len - 1) / len;
  Best* best = static_cast<Best*>(workspace);
  choose_kernel<E><<<dim3((unsigned)parts, (unsigned)a.T, (unsigned)a.B), kChooseThreads, 0, stream>>>(a, best, len);
  walk_kernel<E, kParts, 256><<<(unsigned)a.B, 256, 0, stream>>>(a, best, parts);
}

}  // namespace

// All rows at once where their logits are no more than the card reads in a walk's time, 96 MiB.  Both ways, us, 151936 bf16:
// 2 trees of 65 rows (40 MB) 15 / 25, 4 of 65 (79 MB) 23 - 26 / 42, 1 of 257 (78 MB) 20 - 23 / 24.4.
int verify_parts(int64_t B, int64_t T, int32_t V, size_t elem) {
  const int64_t rows = B * T;
  if (rows < 1 || rows * V * (int64_t)elem > 96 << 20) return 0;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / rows, V / 4096, kWave}));
}
size_t verify_workspace(int64_t B, int64_t T, int32_t V, size_t elem) {
  return (size_t)(B * T * verify_parts(B, T, V, elem)) * sizeof(Best);
}

hipError_t launch_verify(const VerifyArgs& a, void* workspace, caddtree_dtype_t dtype, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) launch<BF16>(a, workspace, 2, stream);
  else if (dtype == CADDTREE_F16) launch<F16>(a, workspace, 2, stream);
  else launch<F32>(a, workspace, 4, stream);
  return hipGetLastError();
}

}  // namespace caddtree
