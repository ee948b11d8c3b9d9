// The Python binding's calls, natively: checks the tensors of a call against the plan, as the Python
// checks do, and calls the library.
//
// A call's checks look at up to thirteen tensors.  Through the tensors' Python attributes they cost more
// than the kernels of a small round: 16 of the 22 us of host time of a build, 30 of the 37 us of the three
// stage calls.  Here a call takes about 1 us besides the launches.
//
// A function returns the library's status, or None when it cannot vouch for every argument: then the
// caller takes the Python path, which decides (and raises) as it always did.  Nothing is kept from one
// call to the next.
#define PY_SSIZE_T_CLEAN
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "caddtree.h"

namespace {

// What the checks need of a plan, and the library's functions (ctypes has loaded them).
struct Spec {
  caddtree_plan_t plan;
  int device;            // GPU index; -1: host tensors (tests of the checks themselves)
  int64_t L, V, K, cap;  // cap at least 1, as the outputs are shaped
  c10::ScalarType dtype;
  int mask;              // caddtree_mask_t
  decltype(&caddtree_build) build;
  decltype(&caddtree_build_noalloc) build_noalloc;
  decltype(&caddtree_reduce_topk) reduce_topk;
  decltype(&caddtree_expand) expand;
  decltype(&caddtree_emit) emit;
  decltype(&caddtree_accept) accept;
};

// One call's view of its arguments: ok falls, and stays down, at the first one that is not as it should be.
struct Call {
  const Spec& s;
  bool ok = true;
  PyObject* held[16];    // attributes fetched from an outputs object, until the call returns
  int n_held = 0;

  explicit Call(const Spec& spec) : s(spec) {}
  ~Call() {
    for (int i = 0; i < n_held; ++i) Py_DECREF(held[i]);
  }
  Call(const Call&) = delete;
  Call& operator=(const Call&) = delete;

  PyObject* attr(PyObject* o, PyObject* name) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (v == nullptr) {
      PyErr_Clear();
      ok = false;
      return Py_None;
    }
    held[n_held++] = v;
    return v;
  }

  // the tensor behind o: exactly a torch.Tensor, strided, with storage, on the plan's device
  c10::TensorImpl* tensor(PyObject* o) {
    if (!ok || !THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    c10::TensorImpl* t = THPVariable_Unpack(o).unsafeGetTensorImpl();
    const c10::Device d = t->device();
    const bool here = s.device >= 0 ? d.is_cuda() && d.index() == s.device : d.is_cpu();
    if (!here || t->layout() != c10::kStrided || !t->has_storage() || t->has_symbolic_sizes_strides()) {
      ok = false;
      return nullptr;
    }
    return t;
  }

  // a contiguous tensor of `type`, shaped [>= B, dims...]; None gives nullptr unless it is required
  void* data(PyObject* o, c10::ScalarType type, std::initializer_list<int64_t> dims, int64_t B, bool required) {
    if (o == Py_None) {
      if (required) ok = false;
      return nullptr;
    }
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr) return nullptr;
    const auto sz = t->sizes();
    bool good = c10::typeMetaToScalarType(t->dtype()) == type && sz.size() == 1 + dims.size() && sz[0] >= B &&
                t->is_contiguous();
    size_t i = 1;
    if (good)
      for (const int64_t d : dims) good = good && sz[i++] == d;
    if (!good || t->numel() == 0) {
      ok = false;
      return nullptr;
    }
    return t->mutable_data();
  }

  // rows (b, i) at element (b L + i) stride
  void* logits(PyObject* o, int64_t* B, int64_t* stride) {
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr) return nullptr;
    const auto sz = t->sizes();
    if (c10::typeMetaToScalarType(t->dtype()) != s.dtype || sz.size() != 3 || sz[1] != s.L || sz[2] < s.V ||
        t->numel() == 0) {
      ok = false;
      return nullptr;
    }
    const auto st = t->strides();
    int64_t rs;
    bool good = true;
    if (s.L > 1) {
      rs = st[1];
      good = sz[0] == 1 || st[0] == rs * s.L;
    } else {
      rs = sz[0] > 1 ? st[0] : sz[2];
    }
    if (sz[2] > 1 && st[2] != 1) good = false;
    if (!good || rs < s.V) {
      ok = false;
      return nullptr;
    }
    *B = sz[0];
    *stride = rs;
    return const_cast<void*>(t->data());
  }

  int64_t rows(PyObject* o) {
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr || t->sizes().empty()) {
      ok = false;
      return 0;
    }
    return t->sizes()[0];
  }

  const int64_t* ctx(PyObject* o, int64_t B) {
    if (o == Py_None) return nullptr;
    void* p = data(o, c10::kLong, {}, B, true);
    if (ok && rows(o) != B) ok = false;
    return static_cast<const int64_t*>(p);
  }

  void* mask(PyObject* o, int64_t B) {
    if (s.mask == CADDTREE_MASK_U8) return data(o, c10::kByte, {s.cap, s.cap}, B, false);
    if (o == Py_None) return nullptr;
    if (s.mask == CADDTREE_MASK_BITS32) {
      c10::TensorImpl* t = tensor(o);
      if (t == nullptr) return nullptr;
      const c10::ScalarType type = c10::typeMetaToScalarType(t->dtype());
      if (type != c10::kInt && type != c10::kUInt32) {
        ok = false;
        return nullptr;
      }
      return data(o, type, {s.cap, (s.cap + 31) / 32}, B, false);
    }
    ok = false;           // a mask for a plan without one: the Python path decides
    return nullptr;
  }

  int64_t integer(PyObject* o, int64_t lo, int64_t hi) {
    int over = 0;
    const long long v = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &over) : lo - 1;
    if (over != 0 || v < lo || v > hi) ok = false;
    return v;
  }
  int32_t offset(PyObject* o) { return (int32_t)integer(o, INT32_MIN, INT32_MAX); }
  hipStream_t stream(PyObject* o) {
    const unsigned long long v = PyLong_CheckExact(o) ? PyLong_AsUnsignedLongLong(o) : 0;
    if (!PyLong_CheckExact(o) || PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return reinterpret_cast<hipStream_t>(static_cast<uintptr_t>(v));
  }
};

// the attributes of an outputs object
enum Field { kTokenIds, kParent, kDepth, kPathProb, kNStar, kPhi, kTheta, kMask, kPosIds, kTopkIds, kTopkLogit,
             kTopkLq, kLse, kFields };
const char* const kNames[kFields] = {"token_ids", "parent", "depth", "path_prob", "n_star", "phi", "theta",
                                     "mask", "pos_ids", "topk_ids", "topk_logit", "topk_lq", "lse"};
PyObject* g_name[kFields];   // interned

template <typename T>
T* as(void* p) { return static_cast<T*>(p); }

const char* const kSpecName = "caddtree.spec";

// an exception came out of the library's call, whose work may be enqueued already: not to be called again
struct LibraryThrew {};

template <typename F>
PyObject* guarded(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, F&& body) {
  if (nargs != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, nargs);
    return nullptr;
  }
  const Spec* s = static_cast<const Spec*>(PyCapsule_GetPointer(args[0], kSpecName));
  if (s == nullptr) return nullptr;
  int status = -1;
  try {
    status = body(*s);
  } catch (const LibraryThrew&) {
    PyErr_SetString(PyExc_RuntimeError, "the caddtree library threw an exception");
    return nullptr;
  } catch (...) {          // a tensor that cannot be looked at this way
    status = -1;
  }
  if (status < 0) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}

// the library's call without the interpreter's lock, as ctypes makes it; the lock is back however the call ends
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
int unlocked(F&& f) {
  try {
    const Unlocked u;
    return (int)f();
  } catch (...) {
    throw LibraryThrew();
  }
}

void tree_fields(Call& c, PyObject* out, int64_t B, caddtree_outputs_t* o) {
  const int64_t cap = c.s.cap;
  o->parent = as<int32_t>(c.data(c.attr(out, g_name[kParent]), c10::kInt, {cap}, B, true));
  o->n_star = as<int32_t>(c.data(c.attr(out, g_name[kNStar]), c10::kInt, {}, B, true));
  o->depth = as<int32_t>(c.data(c.attr(out, g_name[kDepth]), c10::kInt, {cap}, B, true));
  o->token_ids = as<int32_t>(c.data(c.attr(out, g_name[kTokenIds]), c10::kInt, {cap}, B, true));
  o->path_prob = as<float>(c.data(c.attr(out, g_name[kPathProb]), c10::kFloat, {cap}, B, false));
  o->phi = as<float>(c.data(c.attr(out, g_name[kPhi]), c10::kFloat, {}, B, false));
  o->theta = as<float>(c.data(c.attr(out, g_name[kTheta]), c10::kFloat, {}, B, false));
}

void emit_fields(Call& c, PyObject* out, int64_t B, caddtree_outputs_t* o) {
  o->pos_ids = as<int32_t>(c.data(c.attr(out, g_name[kPosIds]), c10::kInt, {c.s.cap}, B, false));
  o->mask = c.mask(c.attr(out, g_name[kMask]), B);
}

void topk_fields(Call& c, PyObject* out, int64_t B, bool required, caddtree_outputs_t* o) {
  const int64_t L = c.s.L, K = c.s.K;
  o->topk_ids = as<int32_t>(c.data(c.attr(out, g_name[kTopkIds]), c10::kInt, {L, K}, B, required));
  o->topk_logit = as<float>(c.data(c.attr(out, g_name[kTopkLogit]), c10::kFloat, {L, K}, B, required));
  o->lse = as<double>(c.data(c.attr(out, g_name[kLse]), c10::kDouble, {L}, B, required));
}

// spec, logits, out, pos_offset, workspace (None for the no-allocation call), ctx_len, stream, noalloc
PyObject* py_build(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 8, [&](const Spec& s) -> int {
    Call c(s);
    int64_t B = 0, stride = 0;
    const void* x = c.logits(a[1], &B, &stride);
    if (!c.ok) return -1;
    caddtree_outputs_t o = {};
    tree_fields(c, a[2], B, &o);
    emit_fields(c, a[2], B, &o);
    topk_fields(c, a[2], B, false, &o);
    o.topk_lq = as<float>(c.data(c.attr(a[2], g_name[kTopkLq]), c10::kFloat, {s.L, s.K}, B, false));
    const int32_t pos = c.offset(a[3]);
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (c.ok && a[4] != Py_None) {
      c10::TensorImpl* t = c.tensor(a[4]);
      if (t == nullptr || !t->is_contiguous() || t->numel() == 0) return -1;
      ws = t->mutable_data();
      ws_bytes = (size_t)t->numel() * t->itemsize();
    }
    const int64_t* ctx = c.ctx(a[5], B);
    const hipStream_t st = c.stream(a[6]);
    if (!c.ok) return -1;
    if (a[7] == Py_True)
      return unlocked([&] { return s.build_noalloc(s.plan, x, B, stride, pos, ctx, &o, st); });
    return unlocked([&] { return s.build(s.plan, x, B, stride, pos, ctx, &o, ws, ws_bytes, st); });
  });
}

// spec, logits, topk_ids, topk_logit, lse, topk_lq, stream
PyObject* py_reduce_topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 7, [&](const Spec& s) -> int {
    Call c(s);
    int64_t B = 0, stride = 0;
    const void* x = c.logits(a[1], &B, &stride);
    if (!c.ok) return -1;
    auto* ids = as<int32_t>(c.data(a[2], c10::kInt, {s.L, s.K}, B, true));
    auto* logit = as<float>(c.data(a[3], c10::kFloat, {s.L, s.K}, B, true));
    auto* lse = as<double>(c.data(a[4], c10::kDouble, {s.L}, B, true));
    auto* lq = as<float>(c.data(a[5], c10::kFloat, {s.L, s.K}, B, false));
    const hipStream_t st = c.stream(a[6]);
    if (!c.ok) return -1;
    return unlocked([&] { return s.reduce_topk(s.plan, x, B, stride, ids, logit, lq, lse, st); });
  });
}

// spec, topk_ids, topk_logit, lse, out, ctx_len, stream
PyObject* py_expand(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 7, [&](const Spec& s) -> int {
    Call c(s);
    const int64_t B = c.rows(a[1]);
    auto* ids = as<int32_t>(c.data(a[1], c10::kInt, {s.L, s.K}, B, true));
    auto* logit = as<float>(c.data(a[2], c10::kFloat, {s.L, s.K}, B, true));
    auto* lse = as<double>(c.data(a[3], c10::kDouble, {s.L}, B, true));
    if (!c.ok) return -1;
    caddtree_outputs_t o = {};
    tree_fields(c, a[4], B, &o);
    const int64_t* ctx = c.ctx(a[5], B);
    const hipStream_t st = c.stream(a[6]);
    if (!c.ok) return -1;
    return unlocked([&] {
      return s.expand(s.plan, ids, logit, lse, B, ctx, o.token_ids, o.parent, o.depth, o.path_prob, o.n_star, o.phi,
                      o.theta, st);
    });
  });
}

// spec, out, pos_offset, stream
PyObject* py_emit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 4, [&](const Spec& s) -> int {
    Call c(s);
    PyObject* par = c.attr(a[1], g_name[kParent]);
    const int64_t B = c.rows(par);
    caddtree_outputs_t o = {};
    o.parent = as<int32_t>(c.data(par, c10::kInt, {s.cap}, B, true));
    o.n_star = as<int32_t>(c.data(c.attr(a[1], g_name[kNStar]), c10::kInt, {}, B, true));
    emit_fields(c, a[1], B, &o);
    o.depth = as<int32_t>(c.data(c.attr(a[1], g_name[kDepth]), c10::kInt, {s.cap}, B, o.pos_ids != nullptr));
    const int32_t pos = c.offset(a[2]);
    const hipStream_t st = c.stream(a[3]);
    if (!c.ok) return -1;
    return unlocked([&] { return s.emit(s.plan, o.parent, o.depth, o.n_star, B, pos, o.mask, o.pos_ids, st); });
  });
}

// spec, topk, tree, u, accept_len, round_cost, ctx_len, stream
PyObject* py_accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 8, [&](const Spec& s) -> int {
    Call c(s);
    PyObject* tok = c.attr(a[2], g_name[kTokenIds]);
    c10::TensorImpl* t = c.tensor(tok);
    if (t == nullptr || t->sizes().size() != 2) return -1;
    const int64_t B = t->sizes()[0], stride = t->sizes()[1];
    if (stride > INT32_MAX) return -1;
    auto* ids = as<int32_t>(c.data(tok, c10::kInt, {stride}, B, true));
    auto* par = as<int32_t>(c.data(c.attr(a[2], g_name[kParent]), c10::kInt, {stride}, B, true));
    auto* ns = as<int32_t>(c.data(c.attr(a[2], g_name[kNStar]), c10::kInt, {}, B, true));
    caddtree_outputs_t o = {};
    topk_fields(c, a[1], B, true, &o);
    auto* u = as<double>(c.data(a[3], c10::kDouble, {s.L}, B, true));
    if (!c.ok || c.rows(a[3]) != B) return -1;
    auto* al = as<int32_t>(c.data(a[4], c10::kInt, {}, B, true));
    auto* rc = as<double>(c.data(a[5], c10::kDouble, {}, B, false));
    const int64_t* ctx = a[5] != Py_None ? c.ctx(a[6], B) : nullptr;
    const hipStream_t st = c.stream(a[7]);
    if (!c.ok) return -1;
    return unlocked([&] {
      return s.accept(s.plan, o.topk_ids, o.topk_logit, o.lse, B, ids, par, (int32_t)stride, ns, u, ctx, al, rc, st);
    });
  });
}

// handle, device, L, V, K, cap, bf16, mask, the addresses of build, build_noalloc, reduce_topk, expand, emit, accept
PyObject* py_spec(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) {
    PyErr_Format(PyExc_TypeError, "14 arguments expected, got %zd", n);
    return nullptr;
  }
  int64_t v[14];
  for (int i = 0; i < 14; ++i) {
    v[i] = (int64_t)PyLong_AsUnsignedLongLongMask(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Spec* s = new Spec();
  s->plan = reinterpret_cast<caddtree_plan_t>(v[0]);
  s->device = (int)v[1];
  s->L = v[2];
  s->V = v[3];
  s->K = v[4];
  s->cap = v[5] > 1 ? v[5] : 1;
  s->dtype = v[6] ? c10::kBFloat16 : c10::kFloat;
  s->mask = (int)v[7];
  s->build = reinterpret_cast<decltype(s->build)>(v[8]);
  s->build_noalloc = reinterpret_cast<decltype(s->build_noalloc)>(v[9]);
  s->reduce_topk = reinterpret_cast<decltype(s->reduce_topk)>(v[10]);
  s->expand = reinterpret_cast<decltype(s->expand)>(v[11]);
  s->emit = reinterpret_cast<decltype(s->emit)>(v[12]);
  s->accept = reinterpret_cast<decltype(s->accept)>(v[13]);
  PyObject* cap = PyCapsule_New(s, kSpecName, [](PyObject* o) {
    delete static_cast<Spec*>(PyCapsule_GetPointer(o, kSpecName));
  });
  if (cap == nullptr) delete s;
  return cap;
}

// ---------------------------------------------------------------- attention and the cache

// The library's functions, and the device of the calls' tensors where it is not a GPU (tests of the checks).
struct Ops {
  bool host;
  decltype(&caddtree_window_attention) window;
  decltype(&caddtree_cache_attention) attention;
  decltype(&caddtree_cache_write) write;
  decltype(&caddtree_cache_read) read;
  decltype(&caddtree_cache_score) score;
  decltype(&caddtree_cache_evict) evict;
};
const char* const kOpsName = "caddtree.ops";
constexpr int64_t kAny = -1;

// One call's view of its arguments, as Call above: ok falls at the first one that is not as it should be.
struct Attn {
  const Ops& s;
  int device;
  bool ok = true;

  Attn(const Ops& ops, PyObject* dev) : s(ops) { device = (int)integer(dev, 0, 1 << 20); }

  c10::TensorImpl* tensor(PyObject* o) {
    if (!ok || !THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    c10::TensorImpl* t = THPVariable_Unpack(o).unsafeGetTensorImpl();
    const c10::Device d = t->device();
    const bool here = s.host ? d.is_cpu() : d.is_cuda() && d.index() == device;
    if (!here || t->layout() != c10::kStrided || !t->has_storage() || t->has_symbolic_sizes_strides() || t->numel() == 0) {
      ok = false;
      return nullptr;
    }
    return t;
  }

  // a contiguous tensor of `type` with exactly these sizes (kAny: any); None gives nullptr unless it is required
  void* array(PyObject* o, c10::ScalarType type, std::initializer_list<int64_t> dims, bool required = true) {
    if (o == Py_None) {
      if (required) ok = false;
      return nullptr;
    }
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr) return nullptr;
    const auto sz = t->sizes();
    bool good = c10::typeMetaToScalarType(t->dtype()) == type && sz.size() == dims.size() && t->is_contiguous();
    size_t i = 0;
    if (good)
      for (const int64_t d : dims) {
        good = good && (d == kAny || sz[i] == d) && sz[i] <= INT32_MAX;
        ++i;
      }
    if (!good) {
      ok = false;
      return nullptr;
    }
    return t->mutable_data();
  }
  int64_t size(PyObject* o, size_t dim) {
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr || t->sizes().size() <= dim) {
      ok = false;
      return 0;
    }
    return t->sizes()[dim];
  }

  // [B, tokens, heads, head_dim] with a unit last stride, 16-byte aligned rows, and for an output no two elements
  // in one place
  caddtree_view_t view(PyObject* o, c10::ScalarType type, const int64_t (&dims)[4], bool output = false) {
    caddtree_view_t v = {nullptr, 0, 0, 0};
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr) return v;
    const auto sz = t->sizes();
    const auto st = t->strides();
    bool good = c10::typeMetaToScalarType(t->dtype()) == type && sz.size() == 4;
    for (int i = 0; good && i < 4; ++i) good = (dims[i] == kAny || sz[i] == dims[i]) && sz[i] <= INT32_MAX;
    if (!good) {
      ok = false;
      return v;
    }
    v.stride_b = sz[0] > 1 ? st[0] : 0;
    v.stride_t = sz[1] > 1 ? st[1] : 0;
    v.stride_h = sz[2] > 1 ? st[2] : 0;
    v.data = output ? t->mutable_data() : const_cast<void*>(t->data());
    if (st[3] != 1 || (v.stride_b | v.stride_t | v.stride_h) % 8 != 0 || reinterpret_cast<uintptr_t>(v.data) % 16 != 0) ok = false;
    if (output) {
      int64_t n[3] = {sz[0], sz[1], sz[2]}, s3[3] = {v.stride_b, v.stride_t, v.stride_h}, room = sz[3];
      for (int pass = 0; pass < 3; ++pass) {        // strides in ascending order, each past the ones before
        int least = -1;
        for (int i = 0; i < 3; ++i)
          if (n[i] > 1 && (least < 0 || s3[i] < s3[least])) least = i;
        if (least < 0) break;
        if (s3[least] < room) ok = false;
        room += s3[least] * (n[least] - 1);
        n[least] = 1;
      }
    }
    return v;
  }

  // attention has no backward pass: an input that wants one is the Python path's to refuse
  void no_gradient(PyObject* o) {
    if (!c10::GradMode::is_enabled()) return;
    const c10::TensorImpl* t = tensor(o);
    if (t != nullptr && t->requires_grad()) ok = false;
  }

  int64_t integer(PyObject* o, int64_t lo, int64_t hi) {
    int over = 0;
    const long long v = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &over) : lo - 1;
    if (over != 0 || v < lo || v > hi) ok = false;
    return v;
  }
  int32_t count(PyObject* o) { return (int32_t)integer(o, 0, INT32_MAX); }
  float scale(PyObject* o, int64_t head_dim) {
    if (o == Py_None) return (float)(1.0 / std::sqrt((double)head_dim));
    if (!PyFloat_CheckExact(o)) ok = false;
    return ok ? (float)PyFloat_AS_DOUBLE(o) : 0.f;
  }
  bool truth(PyObject* o) {
    if (o != Py_True && o != Py_False) ok = false;
    return o == Py_True;
  }
  hipStream_t stream(PyObject* o) {
    const unsigned long long v = PyLong_CheckExact(o) ? PyLong_AsUnsignedLongLong(o) : 0;
    if (!PyLong_CheckExact(o) || PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return reinterpret_cast<hipStream_t>(static_cast<uintptr_t>(v));
  }
  void* workspace(PyObject* o, size_t* bytes) {
    *bytes = 0;
    if (o == Py_None) return nullptr;
    c10::TensorImpl* t = tensor(o);
    if (t == nullptr || !t->is_contiguous()) {
      ok = false;
      return nullptr;
    }
    *bytes = (size_t)t->numel() * t->itemsize();
    return t->mutable_data();
  }
  const caddtree_cache_t* cache(PyObject* o) {      // the address of the cache object's own description
    return reinterpret_cast<const caddtree_cache_t*>(static_cast<uintptr_t>(integer(o, 1, INT64_MAX)));
  }
  c10::ScalarType type(const caddtree_cache_t* c) { return c->dtype == CADDTREE_BF16 ? c10::kBFloat16 : c10::kHalf; }

  // what every attention call says of its queries
  c10::ScalarType queries(PyObject* q, caddtree_attention_t* a) {
    c10::TensorImpl* t = tensor(q);
    if (t == nullptr || t->sizes().size() != 4) {
      ok = false;
      return c10::kFloat;
    }
    const c10::ScalarType type = c10::typeMetaToScalarType(t->dtype());
    if (type != c10::kBFloat16 && type != c10::kHalf) ok = false;
    a->q = view(q, type, {kAny, kAny, kAny, kAny});
    if (!ok) return type;
    a->dtype = type == c10::kBFloat16 ? CADDTREE_BF16 : CADDTREE_F16;
    a->B = (int32_t)t->sizes()[0];
    a->T = (int32_t)t->sizes()[1];
    a->n_heads = (int32_t)t->sizes()[2];
    a->head_dim = (int32_t)t->sizes()[3];
    return type;
  }
  // ... and a call over a cache of its pages, lengths and form
  c10::ScalarType cached(const caddtree_cache_t* c, PyObject* q, PyObject* table, PyObject* ctx, PyObject* cnt, PyObject* depth,
                         PyObject* window, PyObject* sinks, PyObject* sc, caddtree_attention_t* a) {
    const c10::ScalarType t = queries(q, a);
    if (!ok || a->dtype != c->dtype || a->head_dim != c->head_dim) {
      ok = false;
      return t;
    }
    a->n_kv_heads = c->n_kv_heads;
    a->S = a->T;
    a->page_table = as<int32_t>(array(table, c10::kInt, {a->B, kAny}));
    a->ctx_len = as<int64_t>(array(ctx, c10::kLong, {a->B}));
    a->q_len = as<int32_t>(array(cnt, c10::kInt, {a->B}, false));
    if (!ok) return t;
    a->table_pages = (int32_t)size(table, 1);
    if (depth != Py_None) {
      a->depth = as<int32_t>(array(depth, c10::kInt, {a->B, kAny}));
      if (!ok) return t;
      a->cap = (int32_t)size(depth, 1);
      a->order = CADDTREE_ORDER_TREE;
    }
    a->window = count(window);
    a->sinks = count(sinks);
    a->scale = scale(sc, a->head_dim);
    return t;
  }
};

template <typename F>
PyObject* guarded_ops(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, F&& body) {
  if (nargs != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, nargs);
    return nullptr;
  }
  const Ops* s = static_cast<const Ops*>(PyCapsule_GetPointer(args[0], kOpsName));
  if (s == nullptr) return nullptr;
  int status = -1;
  try {
    status = body(*s);
  } catch (const LibraryThrew&) {
    PyErr_SetString(PyExc_RuntimeError, "the caddtree library threw an exception");
    return nullptr;
  } catch (...) {          // a tensor that cannot be looked at this way
    status = -1;
  }
  if (status < 0) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}

// ops, device, stream, q, k, v, window, sinks, causal, scale, q_len, k_len, out, lse, workspace
PyObject* py_window_attention(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 15, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    caddtree_attention_t a = {};
    const c10::ScalarType t = c.queries(p[3], &a);
    if (!c.ok) return -1;
    a.k = c.view(p[4], t, {a.B, kAny, kAny, a.head_dim});
    if (!c.ok) return -1;
    a.S = (int32_t)c.size(p[4], 1);
    a.n_kv_heads = (int32_t)c.size(p[4], 2);
    a.v = c.view(p[5], t, {a.B, a.S, a.n_kv_heads, a.head_dim});
    a.window = c.count(p[6]);
    a.sinks = c.count(p[7]);
    a.order = c.truth(p[8]) ? CADDTREE_ORDER_CHAIN : CADDTREE_ORDER_BLOCK;
    a.scale = c.scale(p[9], a.head_dim);
    a.q_len = as<int32_t>(c.array(p[10], c10::kInt, {a.B}, false));
    a.k_len = as<int32_t>(c.array(p[11], c10::kInt, {a.B}, false));
    a.out = c.view(p[12], t, {a.B, a.T, a.n_heads, a.head_dim}, true);
    a.lse = as<float>(c.array(p[13], c10::kFloat, {a.B, a.T, a.n_heads}, false));
    size_t bytes;
    void* ws = c.workspace(p[14], &bytes);
    for (int i = 3; i < 6; ++i) c.no_gradient(p[i]);
    if (!c.ok) return -1;
    return unlocked([&] { return s.window(&a, ws, bytes, st); });
  });
}

// ops, device, stream, cache, q, page_table, ctx_len, k, v, count, causal, mask, depth, window, sinks, scale, out, lse,
// workspace
PyObject* py_cache_attention(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 19, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    const caddtree_cache_t* cache = c.cache(p[3]);
    if (!c.ok) return -1;
    caddtree_attention_t a = {};
    const c10::ScalarType t = c.cached(cache, p[4], p[5], p[6], p[9], p[12], p[13], p[14], p[15], &a);
    if (!c.ok) return -1;
    const bool causal = c.truth(p[10]), tree = p[12] != Py_None, keys = p[7] != Py_None;
    if (!tree) a.order = causal ? CADDTREE_ORDER_CHAIN : CADDTREE_ORDER_BLOCK;
    if (keys != (p[8] != Py_None) || (p[11] != Py_None && !tree) || (tree && keys && p[11] == Py_None)) return -1;
    if (p[11] != Py_None) {
      c10::TensorImpl* m = c.tensor(p[11]);
      if (m == nullptr) return -1;
      const c10::ScalarType mt = c10::typeMetaToScalarType(m->dtype());
      if (mt == c10::kByte) {
        a.mask_kind = CADDTREE_MASK_U8;
        a.mask = c.array(p[11], mt, {a.B, a.cap, a.cap});
      } else if (mt == c10::kInt || mt == c10::kUInt32) {
        a.mask_kind = CADDTREE_MASK_BITS32;
        a.mask = c.array(p[11], mt, {a.B, a.cap, (a.cap + 31) / 32});
      } else {
        return -1;
      }
    }
    if (keys) {
      a.k = c.view(p[7], t, {a.B, a.T, a.n_kv_heads, a.head_dim});
      a.v = c.view(p[8], t, {a.B, a.T, a.n_kv_heads, a.head_dim});
    }
    a.out = c.view(p[16], t, {a.B, a.T, a.n_heads, a.head_dim}, true);
    a.lse = as<float>(c.array(p[17], c10::kFloat, {a.B, a.T, a.n_heads}, false));
    size_t bytes;
    void* ws = c.workspace(p[18], &bytes);
    c.no_gradient(p[4]);
    if (keys) {
      c.no_gradient(p[7]);
      c.no_gradient(p[8]);
    }
    if (!c.ok) return -1;
    return unlocked([&] { return s.attention(cache, &a, ws, bytes, st); });
  });
}

// ops, device, stream, cache, k, v, page_table, start, count, index
PyObject* py_cache_write(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 10, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    const caddtree_cache_t* cache = c.cache(p[3]);
    if (!c.ok) return -1;
    const int64_t B = c.size(p[6], 0);
    const auto* table = as<int32_t>(c.array(p[6], c10::kInt, {B, kAny}));
    if (!c.ok) return -1;
    const int32_t pages = (int32_t)c.size(p[6], 1);
    const caddtree_view_t k = c.view(p[4], c.type(cache), {B, kAny, cache->n_kv_heads, cache->head_dim});
    if (!c.ok) return -1;
    const int64_t rows = c.size(p[4], 1);
    const caddtree_view_t v = c.view(p[5], c.type(cache), {B, rows, cache->n_kv_heads, cache->head_dim});
    const auto* start = as<int64_t>(c.array(p[7], c10::kLong, {B}));
    const auto* count = as<int32_t>(c.array(p[8], c10::kInt, {B}, false));
    const auto* index = as<int32_t>(c.array(p[9], c10::kInt, {B, kAny}, false));
    if (!c.ok) return -1;
    const int64_t T = index ? c.size(p[9], 1) : rows;
    return unlocked([&] { return s.write(cache, &k, &v, (int32_t)B, (int32_t)T, (int32_t)rows, start, count, index, table, pages, st); });
  });
}

// ops, device, stream, cache, k, v, page_table, start, end
PyObject* py_cache_read(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 9, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    const caddtree_cache_t* cache = c.cache(p[3]);
    if (!c.ok) return -1;
    const int64_t B = c.size(p[6], 0);
    const auto* table = as<int32_t>(c.array(p[6], c10::kInt, {B, kAny}));
    if (!c.ok) return -1;
    const int32_t pages = (int32_t)c.size(p[6], 1);
    const caddtree_view_t k = c.view(p[4], c.type(cache), {B, kAny, cache->n_kv_heads, cache->head_dim}, true);
    if (!c.ok) return -1;
    const int64_t T = c.size(p[4], 1);
    const caddtree_view_t v = c.view(p[5], c.type(cache), {B, T, cache->n_kv_heads, cache->head_dim}, true);
    const auto* start = as<int64_t>(c.array(p[7], c10::kLong, {B}, false));
    const auto* end = as<int64_t>(c.array(p[8], c10::kLong, {B}));
    if (!c.ok) return -1;
    return unlocked([&] { return s.read(cache, &k, &v, (int32_t)B, (int32_t)T, start, end, table, pages, st); });
  });
}

// ops, device, stream, cache, q, page_table, ctx_len, lse, scores, new_scores, weight, count, depth, window, sinks, scale
PyObject* py_cache_score(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 16, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    const caddtree_cache_t* cache = c.cache(p[3]);
    if (!c.ok) return -1;
    caddtree_attention_t a = {};
    c.cached(cache, p[4], p[5], p[6], p[11], p[12], p[13], p[14], p[15], &a);
    if (!c.ok) return -1;
    a.lse = as<float>(c.array(p[7], c10::kFloat, {a.B, a.T, a.n_heads}));
    auto* scores = as<float>(c.array(p[8], c10::kFloat, {a.B, a.n_kv_heads, kAny}));
    if (!c.ok) return -1;
    const int64_t slots = c.size(p[8], 2);
    float* fresh = p[9] == Py_None ? scores : as<float>(c.array(p[9], c10::kFloat, {a.B, a.n_kv_heads, slots}));
    const auto* weight = as<float>(c.array(p[10], c10::kFloat, {a.B, a.T}, false));
    if (!c.ok) return -1;
    return unlocked([&] { return s.score(cache, &a, weight, scores, fresh, slots, st); });
  });
}

// ops, device, stream, cache, page_table, ctx_len, scores, new_table, new_len, new_scores, kept, budget, sinks, recent,
// workspace
PyObject* py_cache_evict(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded_ops(p, n, 15, [&](const Ops& s) -> int {
    Attn c(s, p[1]);
    const hipStream_t st = c.stream(p[2]);
    const caddtree_cache_t* cache = c.cache(p[3]);
    if (!c.ok) return -1;
    const int64_t B = c.size(p[4], 0), H = cache->n_kv_heads;
    const auto* table = as<int32_t>(c.array(p[4], c10::kInt, {B, kAny}));
    const auto* ctx = as<int64_t>(c.array(p[5], c10::kLong, {B}));
    const auto* scores = as<float>(c.array(p[6], c10::kFloat, {B, H, kAny}));
    const auto* to = as<int32_t>(c.array(p[7], c10::kInt, {B, kAny}));
    auto* len = as<int64_t>(c.array(p[8], c10::kLong, {B}));
    auto* fresh = as<float>(c.array(p[9], c10::kFloat, {B, H, kAny}));
    const int32_t budget = c.count(p[11]), sinks = c.count(p[12]), recent = c.count(p[13]);
    auto* kept = as<int32_t>(c.array(p[10], c10::kInt, {B, H, budget}));
    size_t bytes = 0;
    void* ws = c.workspace(p[14], &bytes);
    if (!c.ok) return -1;
    const int64_t pages = c.size(p[4], 1), slots = c.size(p[6], 2), to_pages = c.size(p[7], 1), to_slots = c.size(p[9], 2);
    return unlocked([&] {
      return s.evict(cache, (int32_t)B, table, (int32_t)pages, ctx, scores, slots, budget, sinks, recent, to, (int32_t)to_pages,
                     fresh, to_slots, len, kept, ws, bytes, st);
    });
  });
}

// host, the addresses of window_attention, cache_attention, cache_write, cache_read, cache_score, cache_evict
PyObject* py_ops(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_Format(PyExc_TypeError, "7 arguments expected, got %zd", n);
    return nullptr;
  }
  uint64_t v[7];
  for (int i = 0; i < 7; ++i) {
    v[i] = PyLong_AsUnsignedLongLongMask(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Ops* s = new Ops{v[0] != 0,
                   reinterpret_cast<decltype(Ops::window)>(v[1]),
                   reinterpret_cast<decltype(Ops::attention)>(v[2]),
                   reinterpret_cast<decltype(Ops::write)>(v[3]),
                   reinterpret_cast<decltype(Ops::read)>(v[4]),
                   reinterpret_cast<decltype(Ops::score)>(v[5]),
                   reinterpret_cast<decltype(Ops::evict)>(v[6])};
  PyObject* cap = PyCapsule_New(s, kOpsName, [](PyObject* o) { delete static_cast<Ops*>(PyCapsule_GetPointer(o, kOpsName)); });
  if (cap == nullptr) delete s;
  return cap;
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {CALL(spec), CALL(build), CALL(reduce_topk), CALL(expand), CALL(emit), CALL(accept),
                           CALL(ops), CALL(window_attention), CALL(cache_attention), CALL(cache_write), CALL(cache_read),
                           CALL(cache_score), CALL(cache_evict),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  for (int i = 0; i < kFields; ++i)
    if ((g_name[i] = PyUnicode_InternFromString(kNames[i])) == nullptr) return nullptr;
  return PyModule_Create(&g_module);
}
