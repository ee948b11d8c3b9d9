// Arguments of the kernels on logits (adjust.hip, verify.hip, distill.hip), as the host side fills them in.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "caddtree.h"

namespace caddtree {

struct Rows {
  char* data;
  int64_t b, t;              // strides in elements
};

struct AdjustArgs {
  Rows in, out;
  int32_t B, T, V;
  const int32_t* count;
  const int32_t* history;
  const int32_t* history_len;
  int32_t H;
  const float *repetition, *presence, *frequency;
  const int32_t* bias_ids;
  const float* bias;
  int32_t n_bias;
  const uint32_t* allowed;
  int64_t allowed_b, allowed_t;
  const int32_t* token_ids;
  const int32_t* parent;
  float fill;
};
hipError_t launch_adjust(const AdjustArgs& a, caddtree_dtype_t dtype, bool in_place, hipStream_t stream);

struct VerifyArgs {
  Rows in;                   // data NULL: the tokens are in `chosen`
  int32_t B, T, V;
  const int32_t* chosen;
  const int32_t* token_ids;
  const int32_t* parent;
  const int32_t* count;
  int32_t M;
  int32_t* accepted;
  int32_t* index;
  int32_t* tokens;
  float* weight;
};
// How many parts each row is cut into where all rows are read at once (0: the walk reads those of its path), and the
// workspace for that; elem: bytes of a logit.
int verify_parts(int64_t B, int64_t T, int32_t V, size_t elem);
size_t verify_workspace(int64_t B, int64_t T, int32_t V, size_t elem);
hipError_t launch_verify(const VerifyArgs& a, void* workspace, caddtree_dtype_t dtype, hipStream_t stream);

struct DistillArgs {
  Rows in, grad;             // grad.data NULL: none
  int32_t B, T, V, K;
  const int32_t* ids;
  const float* target;
  const float* weight;
  float c32;                 // log2(e) / temperature, rounded
  double c, inverse;         // ... and 1 / temperature
  double off;                // (c - c32) / c
  int32_t tail;
  float* loss;
  float* stats;
};
// How many parts a row is cut into where there is a workspace, and its bytes (0: one part).
int distill_parts(int64_t rows, int32_t V);
size_t distill_workspace(int64_t rows, int32_t V);
// ... where its gradient is written by itself; elem: bytes of a logit.
int distill_grad_parts(int32_t V, size_t elem);
hipError_t launch_distill(const DistillArgs& a, void* workspace, caddtree_dtype_t dtype, hipStream_t stream);
hipError_t launch_distill_grad(const DistillArgs& a, caddtree_dtype_t dtype, hipStream_t stream);

}  // namespace caddtree
