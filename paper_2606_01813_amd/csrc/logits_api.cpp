// Host side of the calls on logits declared in caddtree.h: argument checks and launches on the caller's stream.

#include <cmath>
#include <cstdint>

#include "apart.h"
#include "logits_args.h"
#include "status.h"

using caddtree::Array;
using caddtree::check_apart;
using caddtree::enum_value;
using caddtree::fail;
using caddtree::hip_fail;
using caddtree::ok;

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int32_t kMaxRows = 1 << 19;              // of a sequence; and sequences

size_t size_of(int dtype) { return dtype == CADDTREE_F32 ? 4 : 2; }

caddtree_status_t check_sizes(int dtype, int32_t B, int32_t T, int32_t V) {
  if (dtype != CADDTREE_F32 && dtype != CADDTREE_BF16 && dtype != CADDTREE_F16)
    return fail(CADDTREE_E_INVALID, "unknown dtype %d", dtype);
  if (B < 0 || T < 0) return fail(CADDTREE_E_INVALID, "B = %d and T = %d must not be negative", B, T);
  if (B > kMaxRows) return fail(CADDTREE_E_UNSUPPORTED, "B = %d exceeds 2^19 sequences", B);
  if (T > kMaxRows) return fail(CADDTREE_E_UNSUPPORTED, "T = %d exceeds 2^19 rows", T);
  if (V < 1) return fail(CADDTREE_E_INVALID, "V = %d must be >= 1", V);
  if (V > CADDTREE_MAX_VOCAB) return fail(CADDTREE_E_UNSUPPORTED, "V = %d exceeds %d", V, CADDTREE_MAX_VOCAB);
  return CADDTREE_OK;
}

// elements from a tensor's first to its last
int64_t extent(const caddtree_rows_t& r, int32_t B, int32_t T, int32_t V) { return (B - 1) * r.stride_b + (T - 1) * r.stride_t + V; }

// rows [B, T, V] with B, T >= 1; an output's share no element
caddtree_status_t check_rows(const char* name, const caddtree_rows_t& r, int dtype, int32_t B, int32_t T, int32_t V, bool output) {
  if (r.data == nullptr) return fail(CADDTREE_E_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(r.data) % size_of(dtype) != 0)
    return fail(CADDTREE_E_INVALID, "%s is not aligned to its elements", name);
  if (r.stride_b < 0 || r.stride_t < 0) return fail(CADDTREE_E_INVALID, "the strides of %s must not be negative", name);
  if (r.stride_b > kMaxStride || r.stride_t > kMaxStride)
    return fail(CADDTREE_E_UNSUPPORTED, "a stride of %s exceeds 2^40 elements", name);
  if (output) {
    const bool t_inside = B <= 1 || T <= 1 || r.stride_t <= r.stride_b;       // the smaller stride first
    const int64_t s0 = t_inside ? r.stride_t : r.stride_b, s1 = t_inside ? r.stride_b : r.stride_t;
    const int64_t n0 = t_inside ? T : B, n1 = t_inside ? B : T;
    const int64_t inner = n0 > 1 ? (n0 - 1) * s0 + V : V;
    if ((n0 > 1 && s0 < V) || (n1 > 1 && s1 < inner))
      return fail(CADDTREE_E_INVALID, "%s must not overlap itself", name);
  }
  return CADDTREE_OK;
}

bool same(const caddtree_rows_t& x, const caddtree_rows_t& y, int32_t B, int32_t T) {
  return x.data == y.data && (B <= 1 || x.stride_b == y.stride_b) && (T <= 1 || x.stride_t == y.stride_t);
}

Array rows_array(const char* name, const caddtree_rows_t& r, int dtype, int32_t B, int32_t T, int32_t V, bool written) {
  return Array{name, r.data, r.data ? (size_t)extent(r, B, T, V) * size_of(dtype) : 0, written};
}
Array array(const char* name, const void* data, size_t bytes, bool written = false) {
  return Array{name, data, data ? bytes : 0, written};
}

caddtree::Rows rows(const caddtree_rows_t& r) { return caddtree::Rows{static_cast<char*>(r.data), r.stride_b, r.stride_t}; }

caddtree_status_t check_workspace(const void* workspace) {
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(CADDTREE_E_WORKSPACE, "workspace must be 256-byte aligned");
  return CADDTREE_OK;
}

caddtree_status_t check_distill(const caddtree_distill_t* a) {
  if (a == nullptr) return fail(CADDTREE_E_INVALID, "the arguments are NULL");
  const caddtree_status_t st = check_sizes(enum_value(a->dtype), a->B, a->T, a->V);
  if (st != CADDTREE_OK) return st;
  if (a->K < 1) return fail(CADDTREE_E_INVALID, "K = %d must be >= 1", a->K);
  if (a->K > CADDTREE_MAX_TEACHER) return fail(CADDTREE_E_UNSUPPORTED, "K = %d exceeds %d", a->K, CADDTREE_MAX_TEACHER);
  if (!(a->temperature >= 0x1p-20f && a->temperature <= 0x1p20f))
    return fail(CADDTREE_E_INVALID, "temperature = %g must be in 2^-20 .. 2^20", a->temperature);
  if (a->tail != 0 && a->tail != 1) return fail(CADDTREE_E_INVALID, "tail = %d must be 0 or 1", a->tail);
  return CADDTREE_OK;
}

caddtree::DistillArgs distill_args(const caddtree_distill_t* a) {
  const double c = 0x1.71547652b82fep+0 / (double)a->temperature;             // log2(e) / temperature
  return caddtree::DistillArgs{rows(a->logits), rows(a->grad), a->B, a->T, a->V, a->K, a->ids, a->target, a->weight,
                               (float)c, c, 1.0 / (double)a->temperature, (c - (double)(float)c) / c, a->tail, a->loss, a->stats};
}

// what both distillation calls read, and the gradient
caddtree_status_t check_distill_data(const caddtree_distill_t* a, bool loss, const void* workspace, size_t workspace_bytes) {
  const int dtype = enum_value(a->dtype);
  caddtree_status_t st = check_rows("logits", a->logits, dtype, a->B, a->T, a->V, false);
  if (st != CADDTREE_OK) return st;
  if (a->ids == nullptr || a->target == nullptr) return fail(CADDTREE_E_INVALID, "ids and target are required");
  if (a->grad.data != nullptr || !loss)
    if ((st = check_rows("grad", a->grad, dtype, a->B, a->T, a->V, true)) != CADDTREE_OK) return st;
  const bool in_place = a->grad.data != nullptr && same(a->grad, a->logits, a->B, a->T);
  const size_t n = (size_t)a->B * a->T;
  const Array arrays[] = {rows_array("logits", a->logits, dtype, a->B, a->T, a->V, false),
                          in_place ? array("grad", nullptr, 0) : rows_array("grad", a->grad, dtype, a->B, a->T, a->V, true),
                          array("ids", a->ids, n * a->K * 4), array("target", a->target, n * a->K * 4),
                          array("weight", a->weight, n * 4), array("loss", loss ? a->loss : nullptr, n * 4, true),
                          array("stats", a->stats, n * 12, loss), array("workspace", workspace, workspace_bytes, true)};   // (as far as it is used)
  if ((st = check_apart(arrays)) != CADDTREE_OK) return st;
  if (!in_place) return CADDTREE_OK;
  Array over[8];
  for (int i = 0; i < 8; ++i) over[i] = arrays[i];
  over[0].written = true;                            // (the gradient, over the logits)
  return check_apart(over);
}

}  // namespace

extern "C" {

caddtree_status_t caddtree_adjust_logits(const caddtree_adjust_t* a, hipStream_t stream) {
  if (a == nullptr) return fail(CADDTREE_E_INVALID, "the arguments are NULL");
  const int dtype = enum_value(a->dtype);
  caddtree_status_t st = check_sizes(dtype, a->B, a->T, a->V);
  if (st != CADDTREE_OK) return st;
  if (a->H < 0 || a->n_bias < 0) return fail(CADDTREE_E_INVALID, "H = %d and n_bias = %d must not be negative", a->H, a->n_bias);
  if (a->H > CADDTREE_MAX_HISTORY) return fail(CADDTREE_E_UNSUPPORTED, "H = %d exceeds %d", a->H, CADDTREE_MAX_HISTORY);
  if (a->n_bias > CADDTREE_MAX_BIAS) return fail(CADDTREE_E_UNSUPPORTED, "n_bias = %d exceeds %d", a->n_bias, CADDTREE_MAX_BIAS);
  // (workgroups of 512 threads, for 2 rows of 8192 tokens each, are numbered in 32 bits by their threads)
  if (((int64_t)a->T / 2 + 1) * ((int64_t)a->V / 8192 + 1) >= 1 << 23)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d rows of V = %d: more than 2^23 workgroups", a->T, a->V);
  if (std::isnan(a->fill)) return fail(CADDTREE_E_INVALID, "fill is NaN");
  if (a->B == 0 || a->T == 0) return ok();
  if (a->n_bias > 0 && (a->bias_ids == nullptr || a->bias == nullptr))
    return fail(CADDTREE_E_INVALID, "bias_ids and bias are required with n_bias = %d", a->n_bias);
  if ((a->token_ids == nullptr) != (a->parent == nullptr) && a->T > 1)
    return fail(CADDTREE_E_INVALID, "a tree needs token_ids and parent");
  if (a->parent != nullptr && a->T > CADDTREE_MAX_CAP + 1)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d exceeds a tree of %d nodes and its root", a->T, CADDTREE_MAX_CAP);
  if (reinterpret_cast<uintptr_t>(a->allowed) % 4 != 0) return fail(CADDTREE_E_INVALID, "allowed must be 4-byte aligned");
  if (a->allowed_stride_b < 0 || a->allowed_stride_t < 0 || a->allowed_stride_b > kMaxStride || a->allowed_stride_t > kMaxStride)
    return fail(CADDTREE_E_INVALID, "the strides of allowed must be in 0 .. 2^40 words");
  if ((st = check_rows("logits", a->logits, dtype, a->B, a->T, a->V, false)) != CADDTREE_OK) return st;
  if ((st = check_rows("out", a->out, dtype, a->B, a->T, a->V, true)) != CADDTREE_OK) return st;
  const bool in_place = same(a->out, a->logits, a->B, a->T);
  const size_t B = (size_t)a->B, nodes = (size_t)a->T - 1;
  const caddtree_rows_t mask = {const_cast<void*>(a->allowed), a->allowed_stride_b, a->allowed_stride_t};
  const Array arrays[] = {rows_array("out", a->out, dtype, a->B, a->T, a->V, true),
                          in_place ? array("logits", nullptr, 0) : rows_array("logits", a->logits, dtype, a->B, a->T, a->V, false),
                          array("count", a->count, B * 4),
                          array("history", a->history, B * a->H * 4),
                          array("history_len", a->history_len, B * 4),
                          array("repetition", a->repetition, B * 4),
                          array("presence", a->presence, B * 4),
                          array("frequency", a->frequency, B * 4),
                          array("bias_ids", a->bias_ids, B * a->n_bias * 4),
                          array("bias", a->bias, B * a->n_bias * 4),
                          array("allowed", a->allowed, a->allowed ? (size_t)extent(mask, a->B, a->T, (a->V + 31) / 32) * 4 : 0),
                          array("token_ids", a->token_ids, B * nodes * 4),
                          array("parent", a->parent, B * nodes * 4)};
  if ((st = check_apart(arrays)) != CADDTREE_OK) return st;
  const caddtree::AdjustArgs k = {rows(a->logits), rows(a->out), a->B, a->T, a->V, a->count, a->H > 0 ? a->history : nullptr,
                                  a->history_len, a->H, a->repetition, a->presence, a->frequency, a->bias_ids, a->bias, a->n_bias,
                                  static_cast<const uint32_t*>(a->allowed), a->allowed_stride_b, a->allowed_stride_t,
                                  a->token_ids, a->parent, a->fill == 0.f ? -INFINITY : a->fill};
  const hipError_t e = caddtree::launch_adjust(k, (caddtree_dtype_t)dtype, in_place, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "adjust launch");
}

size_t caddtree_verify_workspace_bytes(const caddtree_verify_t* a) {
  if (a == nullptr || check_sizes(enum_value(a->dtype), a->B, a->T, a->V) != CADDTREE_OK || a->T > CADDTREE_MAX_CAP + 1) return 0;
  return caddtree::verify_workspace(a->B, a->T, a->V, size_of(enum_value(a->dtype)));
}

caddtree_status_t caddtree_verify_tree(const caddtree_verify_t* a, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (a == nullptr) return fail(CADDTREE_E_INVALID, "the arguments are NULL");
  const int dtype = enum_value(a->dtype);
  caddtree_status_t st = check_sizes(dtype, a->B, a->T, a->V);
  if (st != CADDTREE_OK) return st;
  if (a->T < 1) return fail(CADDTREE_E_INVALID, "T = %d rows hold no root", a->T);
  if (a->T > CADDTREE_MAX_CAP + 1)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d exceeds a tree of %d nodes and its root", a->T, CADDTREE_MAX_CAP);
  if (a->M < 1) return fail(CADDTREE_E_INVALID, "M = %d must be >= 1", a->M);
  if ((st = check_workspace(workspace)) != CADDTREE_OK) return st;
  if (a->B == 0) return ok();
  if (a->count == nullptr || (a->T > 1 && (a->token_ids == nullptr || a->parent == nullptr)))
    return fail(CADDTREE_E_INVALID, "token_ids, parent and count are required");
  if (a->accepted == nullptr || a->index == nullptr || a->tokens == nullptr)
    return fail(CADDTREE_E_INVALID, "accepted, index and tokens are required");
  if ((a->logits.data != nullptr) == (a->chosen != nullptr))
    return fail(CADDTREE_E_INVALID, "either logits or chosen is given");
  if (a->logits.data != nullptr)
    if ((st = check_rows("logits", a->logits, dtype, a->B, a->T, a->V, false)) != CADDTREE_OK) return st;
  const size_t need = caddtree_verify_workspace_bytes(a), B = (size_t)a->B, nodes = (size_t)a->T - 1;
  const bool all = need > 0 && workspace != nullptr && workspace_bytes >= need && a->logits.data != nullptr;
  const Array arrays[] = {rows_array("logits", a->logits, dtype, a->B, a->T, a->V, false),
                          array("chosen", a->chosen, B * a->T * 4),
                          array("token_ids", a->token_ids, B * nodes * 4),
                          array("parent", a->parent, B * nodes * 4),
                          array("count", a->count, B * 4),
                          array("accepted", a->accepted, B * 4, true),
                          array("index", a->index, B * a->M * 4, true),
                          array("tokens", a->tokens, B * a->M * 4, true),
                          array("weight", a->weight, B * a->T * 4, true),
                          array("workspace", all ? workspace : nullptr, need, true)};
  if ((st = check_apart(arrays)) != CADDTREE_OK) return st;
  const caddtree::VerifyArgs k = {rows(a->logits), a->B, a->T, a->V, a->chosen, a->token_ids, a->parent, a->count, a->M,
                                  a->accepted, a->index, a->tokens, a->weight};
  const hipError_t e = caddtree::launch_verify(k, all ? workspace : nullptr, (caddtree_dtype_t)dtype, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "verify launch");
}

size_t caddtree_distill_workspace_bytes(const caddtree_distill_t* a) {
  if (a == nullptr || check_sizes(enum_value(a->dtype), a->B, a->T, a->V) != CADDTREE_OK) return 0;
  return caddtree::distill_workspace((int64_t)a->B * a->T, a->V);
}

caddtree_status_t caddtree_distill(const caddtree_distill_t* a, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  caddtree_status_t st = check_distill(a);
  if (st != CADDTREE_OK) return st;
  if ((st = check_workspace(workspace)) != CADDTREE_OK) return st;
  if (a->B == 0 || a->T == 0) return ok();
  if (a->loss == nullptr) return fail(CADDTREE_E_INVALID, "loss is NULL");
  const size_t need = caddtree_distill_workspace_bytes(a);
  void* ws = need > 0 && workspace_bytes >= need ? workspace : nullptr;
  if ((st = check_distill_data(a, true, ws, need)) != CADDTREE_OK) return st;
  const hipError_t e = caddtree::launch_distill(distill_args(a), ws, (caddtree_dtype_t)enum_value(a->dtype), stream);
  return e == hipSuccess ? ok() : hip_fail(e, "distill launch");
}

caddtree_status_t caddtree_distill_grad(const caddtree_distill_t* a, hipStream_t stream) {
  caddtree_status_t st = check_distill(a);
  if (st != CADDTREE_OK) return st;
  // (workgroups of 256 threads are numbered in 32 bits by their threads)
  if ((int64_t)a->T * caddtree::distill_grad_parts(a->V, size_of(enum_value(a->dtype))) >= 1 << 24)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d rows of V = %d: more than 2^24 workgroups", a->T, a->V);
  if (a->B == 0 || a->T == 0) return ok();
  if (a->stats == nullptr) return fail(CADDTREE_E_INVALID, "stats is NULL");
  if ((st = check_distill_data(a, false, nullptr, 0)) != CADDTREE_OK) return st;
  const hipError_t e = caddtree::launch_distill_grad(distill_args(a), (caddtree_dtype_t)enum_value(a->dtype), stream);
  return e == hipSuccess ? ok() : hip_fail(e, "distill gradient launch");
}

}  // extern "C"
