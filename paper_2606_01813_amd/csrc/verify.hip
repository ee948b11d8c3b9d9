// The target's choice along a built tree: from the root's row on, the largest logit's token (of equals the lowest), then
// the child that carries it, until there is none.  The accepted path is what the target would have written by itself.
//
// Only the rows on the path decide, a handful of a tree's hundreds, and which they are is known one row at a time: a
// workgroup walks a tree and reads a row whenever it gets there.  Where all rows of the call are few, that chain is
// longer than reading them all at once: choose_kernel does so, a part of a row a workgroup, and the walk joins the parts.
//
// 32 trees of up to 256 nodes, 151936 bf16 logits a row, take 41 us: the longest path's 9 rows one after the other, 4.4 us each,
// of which a compute unit at 64 bytes a clock needs 2 for the 304 KB and the first loads' latency, the joins and the search for
// the child the rest.  One tree of 64 nodes: 10 us, all rows at once in 6.0 and the walk over the parts in 4.0.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "logits_common.h"

namespace caddtree {
namespace {

using namespace lg;

constexpr int kChooseThreads = 256;
constexpr int kNodes = 2048;                      // of a tree, in LDS (further ones are read where they lie)
constexpr int kAllRows = 520;                     // of a call that reads them all at once, at most

// A row's or a part's choice: the largest logit and the lowest token that has it; none: (-inf, INT_MAX)
struct Best {
  float x;
  int id;
  __device__ __forceinline__ int token() const { return x > -INFINITY ? id : -1; }
  // as a number that is larger for the better (-0 and 0 are equals)
  __device__ __forceinline__ uint64_t key() const {
    const uint32_t w = __float_as_uint(x + 0.f);
    return (uint64_t)(w >> 31 ? ~w : w | 1u << 31) << 32 | ~(uint32_t)id;
  }
};
constexpr uint64_t kNoKey = (uint64_t)0x00800000u << 32;      // (keys of -inf are below)

// A NaN is never chosen, a signalling one neither: outside the mode that a kernel starts in (MODE.IEEE, bit 9 of register 1) the
// maximum of a number and any NaN is the number.  In it a signalling one makes the maximum a NaN, and the next maximum drops
// that with all before it; quieting each logit first would be 8 instructions a vector on top of 13.
__device__ __forceinline__ void numbers_over_nan() { __builtin_amdgcn_s_setreg(1 | 9 << 6, 0); }

// The best of a row's tokens first .. last - 1 (first a multiple of 8) by a workgroup, kU loads in flight a lane.  A lane
// keeps its largest logit and which kU vectors it was among, the first of equals; the lanes that have the workgroup's
// largest read theirs again and look for its token: 13 instructions a vector of 8 logits, of which unpacking is 8.
// s_top and s_id: in LDS, not read any more by a thread that another's call may overtake.
// The walk over 32 trees with 2 / 3 / 4 / 5 loads a lane: 43.4 / 42.1 / 45.2 / 46.3 us (a wavefront's last ones reach past
// the row); 512 threads with 6 45.2.
template <typename E, int kThreads, int kU>
__device__ Best best_of(const typename E::T* row, int first, int last, float* s_top, int* s_id) {
  constexpr int N = kN<E>, kWaves = kThreads / kWave;
  const int n = last / N, tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int edge = n * N + tid;
  const float rest = edge < last && tid < N ? (float)row[edge] : -INFINITY;
  int at = first / N + wave * kWave, got = -1;          // (at: of the wavefront's first lane)
  float top = -INFINITY;
  if (at < n) {
    const uint32_t end = (uint32_t)(n - 1) * 16u;       // (past it a lane sees the last vector again)
    uint32_t byte = (uint32_t)(first / N + tid) * 16u;
    Vec<E> q[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) q[u] = Vec<E>::load_at(row, min(byte + u * kThreads * 16u, end));
    const auto look = [&](bool more) {                  // (inlined for each)
      float t = -INFINITY;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        float x[N];
        __builtin_amdgcn_sched_barrier(0);              // (one vector unpacked at a time: registers)
        q[u].get(x);
#pragma unroll
        for (int j = 0; j < N; ++j) t = fmaxf(t, x[j]);
        if (more) q[u] = Vec<E>::load_at(row, min(byte + u * kThreads * 16u, end));
      }
      const bool up = t > top;
      top = up ? t : top;
      got = up ? at : got;
    };
    for (; at + kU * kThreads < n; at += kU * kThreads) {
      byte += kU * kThreads * 16u;
      look(true);
    }
    look(false);
  }
  const float most = wave_max(fmaxf(top, rest));
  if (tid % kWave == 0) s_top[wave] = most;
  if (tid == 0) *s_id = INT_MAX;
  __syncthreads();
  float x = s_top[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) x = fmaxf(x, s_top[w]);
  if (x > -INFINITY && (top == x || rest == x)) {
    int id = edge;
    if (top == x) {
      const int v = got + tid % kWave;
      Vec<E> q[kU];
      int place = 0;
#pragma unroll
      for (int u = 0; u < kU; ++u) q[u] = row_vector<E>(row, v + u * kThreads, n);
#pragma unroll
      for (int u = kU - 1; u >= 0; --u) {               // (the last first: the lowest of equals stays)
        float y[N];
        q[u].get(y);
#pragma unroll
        for (int j = N - 1; j >= 0; --j) place = y[j] == x ? u * N + j : place;
      }
      id = min(v + place / N * kThreads, n - 1) * N + place % N;
    }
    atomicMin(s_id, id);
  }
  __syncthreads();
  return Best{x, *s_id};
}

// Part blockIdx.x of row blockIdx.y of tree blockIdx.z: parts [B, T, n], of len tokens (a multiple of 8)
template <typename E>
__global__ __launch_bounds__(kChooseThreads) void choose_kernel(VerifyArgs a, Best* parts, int len) {
  __shared__ float s_top[kChooseThreads / kWave];
  __shared__ int s_id;
  numbers_over_nan();
  const int b = (int)blockIdx.z, t = (int)blockIdx.y, first = (int)blockIdx.x * len;
  if (t > min(max(a.count[b], 0), a.T - 1)) return;
  const Best m = best_of<E, kChooseThreads, 4>(row_of<E>(a.in, b, t), first, min(first + len, a.V), s_top, &s_id);
  if (threadIdx.x == 0) parts[((int64_t)b * a.T + t) * gridDim.x + blockIdx.x] = m;
}

enum Source { kRead, kParts, kChosen };               // where a row's token comes from: its logits, their parts, the caller
template <typename E, Source kFrom, int kThreads>
__global__ __launch_bounds__(kThreads) void walk_kernel(VerifyArgs a, const Best* parts, int n_parts) {
  __shared__ float s_top[kThreads / kWave];
  __shared__ int s_id;
  __shared__ uint32_t s_token[kNodes];
  __shared__ uint16_t s_parent[kNodes];               // + 1
  __shared__ int s_child;
  __shared__ uint64_t s_key[kFrom == kParts ? kAllRows : 1]; // of each row
  __shared__ int s_chosen[kFrom == kChosen ? kNodes : 1];
  numbers_over_nan();
  const int b = (int)blockIdx.x, tid = threadIdx.x;
  const int n = min(max(a.count[b], 0), a.T - 1);
  const int32_t* tok = a.token_ids + (int64_t)b * (a.T - 1);
  const int32_t* par = a.parent + (int64_t)b * (a.T - 1);
  if constexpr (kFrom == kParts) {
    for (int i = tid; i < a.T; i += kThreads) s_key[i] = 0;
    __syncthreads();
    for (int i = tid; i < a.T * n_parts; i += kThreads)
      atomicMax(reinterpret_cast<unsigned long long*>(&s_key[i / n_parts]), (unsigned long long)parts[(int64_t)b * a.T * n_parts + i].key());
  }
  if constexpr (kFrom == kChosen)
    for (int i = tid; i < min(a.T, kNodes); i += kThreads) s_chosen[i] = a.chosen[(int64_t)b * a.T + i];
  for (int i = tid; i < min(a.T - 1, kNodes); i += kThreads) {    // (those past n are not looked at)
    const int p = par[i];
    s_token[i] = (uint32_t)tok[i];
    s_parent[i] = (uint16_t)(p >= -1 && p < i ? p + 1 : 0xffff);     // (no child of any row: children come after their parent)
  }
  if (a.weight)
    for (int i = tid; i < a.T; i += kThreads) a.weight[(int64_t)b * a.T + i] = 0.f;
  int row = 0, steps = 0;
  while (true) {
    int t;
    if constexpr (kFrom == kRead) t = best_of<E, kThreads, 3>(row_of<E>(a.in, b, row), 0, a.V, s_top, &s_id).token();
    if (tid == 0) s_child = INT_MAX;
    __syncthreads();                                  // (the weights are cleared too, and what is in LDS is there)
    if constexpr (kFrom == kParts) t = s_key[row] >= kNoKey ? (int)~(uint32_t)s_key[row] : -1;
    if constexpr (kFrom == kChosen) t = row < kNodes ? s_chosen[row] : a.chosen[(int64_t)b * a.T + row];
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
    const int child = __builtin_amdgcn_readfirstlane(s_child);
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
    // (512 or 1024 threads, us: 64 x 65 rows of 8192 bf16 11.5 / 13.7, 16 x 65 of 32000 14.5 / 17.5, 4 x 65 of 65536 19.0 / 19.7,
    // 32 x 257 of 151936 52.5 / 41.3)
    if ((int64_t)a.V * (int64_t)elem <= 128 << 10) walk_kernel<E, kRead, 512><<<(unsigned)a.B, 512, 0, stream>>>(a, nullptr, 0);
    else walk_kernel<E, kRead, 1024><<<(unsigned)a.B, 1024, 0, stream>>>(a, nullptr, 0);
    return;
  }
  const int len = ((a.V + n - 1) / n + 7) & ~7;
  const int parts = (a.V + len - 1) / len;
  Best* best = static_cast<Best*>(workspace);
  choose_kernel<E><<<dim3((unsigned)parts, (unsigned)a.T, (unsigned)a.B), kChooseThreads, 0, stream>>>(a, best, len);
  walk_kernel<E, kParts, 256><<<(unsigned)a.B, 256, 0, stream>>>(a, best, parts);
}

}  // namespace

// All rows at once where they are few: it reads them all, and a walk those of its longest path one after the other, which is not
// known before.  Walk or all, us, bf16, trees x rows of tokens:
//     1 x 65 of 151936 17.4 / 9.5    4 x 65 of 151936 31.5 / 19.1    1 x 257 of 151936 17.3 / 18.0   8 x 65 of 151936 31.5 / 37.2
//     1 x 65 of 32000 9.0 / 8.2      4 x 65 of 65536 19.0 / 13.1     8 x 65 of 65536 19.1 / 18.4
//     1 x 513 of 32000 9.2 / 13.5    1 x 513 of 1024 6.8 / 9.7       64 x 65 of 8192 11.5 / 18.0     64 x 513 of 1024 15.4 / 45.0
int verify_parts(int64_t B, int64_t T, int32_t V, size_t elem) {
  const int64_t rows = B * T;
  if (rows < 1 || rows > kAllRows || rows * V * (int64_t)elem > 96 << 20) return 0;
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
