// Host side of the attention and cache calls declared in caddtree.h: argument checks and launches on the
// caller's stream.

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "attn_args.h"
#include "status.h"

using caddtree::enum_value;
using caddtree::fail;
using caddtree::hip_fail;
using caddtree::ok;

namespace {

using caddtree::AttnArgs;
using caddtree::PagedKV;
using caddtree::View;

constexpr int kResident = 512;                     // workgroups of the attention kernels on the card at a time
constexpr int64_t kMaxStride = (int64_t)1 << 24;   // of a token: 64 of them stay within 2^31 bytes
constexpr int64_t kMaxTokens = (int64_t)1 << 30;   // positions, and the tokens of a table, stay within int32

caddtree_status_t check_type(int dtype, int32_t head_dim) {
  if (dtype == CADDTREE_F32) return fail(CADDTREE_E_UNSUPPORTED, "dtype F32 is not supported here: BF16 or F16");
  if (dtype != CADDTREE_BF16 && dtype != CADDTREE_F16) return fail(CADDTREE_E_INVALID, "unknown dtype %d", dtype);
  if (head_dim < 1) return fail(CADDTREE_E_INVALID, "head_dim = %d must be >= 1", head_dim);
  if (head_dim != 64 && head_dim != 128)
    return fail(CADDTREE_E_UNSUPPORTED, "head_dim = %d: only 64 and 128 are supported", head_dim);
  return CADDTREE_OK;
}

caddtree_status_t check_view(const char* name, const caddtree_view_t& v, bool required) {
  if (v.data == nullptr) return required ? fail(CADDTREE_E_INVALID, "%s is NULL", name) : CADDTREE_OK;
  if (reinterpret_cast<uintptr_t>(v.data) % 16 != 0) return fail(CADDTREE_E_INVALID, "%s must be 16-byte aligned", name);
  if (v.stride_b < 0 || v.stride_t < 0 || v.stride_h < 0 || v.stride_b % 8 != 0 || v.stride_t % 8 != 0 || v.stride_h % 8 != 0)
    return fail(CADDTREE_E_INVALID, "the strides of %s must be multiples of 8 elements, and not negative", name);
  if (v.stride_t >= kMaxStride)
    return fail(CADDTREE_E_UNSUPPORTED, "stride_t = %lld of %s exceeds 2^24 elements", (long long)v.stride_t, name);
  return CADDTREE_OK;
}

caddtree_status_t check_cache(const caddtree_cache_t* c) {
  if (c == nullptr) return fail(CADDTREE_E_INVALID, "cache is NULL");
  const caddtree_status_t st = check_type(enum_value(c->dtype), c->head_dim);
  if (st != CADDTREE_OK) return st;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535)
    return fail(CADDTREE_E_INVALID, "n_kv_heads = %d must be in 1 .. 65535", c->n_kv_heads);
  if (c->n_pages < 0 || c->n_pages > INT32_MAX)
    return fail(CADDTREE_E_INVALID, "n_pages = %lld must be in 0 .. 2^31 - 1", (long long)c->n_pages);
  if (c->pages == nullptr) return fail(CADDTREE_E_INVALID, "the cache's pages are NULL");
  if (reinterpret_cast<uintptr_t>(c->pages) % 256 != 0)
    return fail(CADDTREE_E_INVALID, "the cache's pages must be 256-byte aligned");
  return CADDTREE_OK;
}

caddtree_status_t check_table(const char* name, const int32_t* table, int32_t pages) {
  if (pages < 0 || (int64_t)pages * CADDTREE_PAGE > kMaxTokens)
    return fail(CADDTREE_E_INVALID, "%s: %d pages a sequence, 0 .. 2^30 / %d are possible", name, pages, CADDTREE_PAGE);
  if (table == nullptr && pages > 0) return fail(CADDTREE_E_INVALID, "%s is NULL", name);
  return CADDTREE_OK;
}

caddtree_status_t check_batch(int32_t B) {
  if (B < 0) return fail(CADDTREE_E_INVALID, "B = %d is negative", B);
  if (B > 65535) return fail(CADDTREE_E_UNSUPPORTED, "B = %d exceeds 65535", B);
  return CADDTREE_OK;
}

View view(const caddtree_view_t& v) { return View{static_cast<char*>(v.data), v.stride_b, v.stride_t, v.stride_h}; }

PagedKV paged(const caddtree_cache_t* c, const int32_t* table, int32_t pages) {
  return PagedKV{static_cast<uint8_t*>(c->pages), c->n_pages, table, pages, c->n_kv_heads,
                 (int32_t)CADDTREE_PAGE_BYTES(c->head_dim)};
}

// The sizes of a call, which its workspace depends on.
caddtree_status_t check_sizes(const caddtree_attention_t* a) {
  if (a == nullptr) return fail(CADDTREE_E_INVALID, "the attention arguments are NULL");
  caddtree_status_t st = check_type(enum_value(a->dtype), a->head_dim);
  if (st != CADDTREE_OK) return st;
  if ((st = check_batch(a->B)) != CADDTREE_OK) return st;
  if (a->T < 0 || a->S < 0) return fail(CADDTREE_E_INVALID, "T = %d and S = %d must not be negative", a->T, a->S);
  if (a->n_kv_heads < 1 || a->n_heads < 1 || a->n_heads % a->n_kv_heads != 0)
    return fail(CADDTREE_E_INVALID, "n_heads = %d must be a positive multiple of n_kv_heads = %d", a->n_heads, a->n_kv_heads);
  if (a->n_heads > 65535) return fail(CADDTREE_E_UNSUPPORTED, "n_heads = %d exceeds 65535", a->n_heads);
  if (a->T > kMaxTokens || a->S > kMaxTokens || (int64_t)a->T * (a->n_heads / a->n_kv_heads) > kMaxTokens)
    return fail(CADDTREE_E_UNSUPPORTED, "more than 2^30 tokens, or rows of a kv head, in a sequence");
  // (workgroups are numbered in 31 bits: one for 128 rows, or for 8 kv heads at least)
  if (((int64_t)a->T * (a->n_heads / a->n_kv_heads) / 128 + 1) * ((int64_t)a->B * a->n_kv_heads + 8) > kMaxTokens)
    return fail(CADDTREE_E_UNSUPPORTED, "more than 2^30 workgroups of 128 rows in a call");
  if (a->window < 0 || a->sinks < 0)
    return fail(CADDTREE_E_INVALID, "window = %d and sinks = %d must not be negative", a->window, a->sinks);
  return CADDTREE_OK;
}

// What every attention call and the scores share; the tensors that a call reads are checked by it.
caddtree_status_t check_attention(const caddtree_attention_t* a, const caddtree_cache_t* cache) {
  caddtree_status_t st = check_sizes(a);
  if (st != CADDTREE_OK) return st;
  if (!std::isfinite(a->scale)) return fail(CADDTREE_E_INVALID, "scale must be finite");
  if (std::fabs(a->scale) > 0x1p127f)               // (its product with log2(e) is a float)
    return fail(CADDTREE_E_UNSUPPORTED, "scale = %g: more than 2^127 in magnitude is not supported", a->scale);
  const int order = enum_value(a->order), mask = enum_value(a->mask_kind);
  if (order != CADDTREE_ORDER_CHAIN && order != CADDTREE_ORDER_BLOCK && order != CADDTREE_ORDER_TREE)
    return fail(CADDTREE_E_INVALID, "unknown order %d", order);
  if (order == CADDTREE_ORDER_TREE) {
    if (cache == nullptr) return fail(CADDTREE_E_INVALID, "a tree's attention reads a cache");
    if (mask != CADDTREE_MASK_NONE && mask != CADDTREE_MASK_U8 && mask != CADDTREE_MASK_BITS32)
      return fail(CADDTREE_E_INVALID, "unknown mask kind %d", mask);
    if (a->cap < 0 || a->cap > CADDTREE_MAX_CAP || a->T > a->cap + 1)
      return fail(CADDTREE_E_INVALID, "T = %d queries do not fit a tree of cap = %d nodes and its root", a->T, a->cap);
    if (a->T > 1 && a->depth == nullptr) return fail(CADDTREE_E_INVALID, "a tree needs depth");
  }
  if (cache != nullptr) {
    if ((st = check_cache(cache)) != CADDTREE_OK) return st;
    if (enum_value(cache->dtype) != enum_value(a->dtype) || cache->n_kv_heads != a->n_kv_heads ||
        cache->head_dim != a->head_dim)
      return fail(CADDTREE_E_INVALID, "the cache's dtype, n_kv_heads or head_dim is not the call's");
    if ((st = check_table("page_table", a->page_table, a->table_pages)) != CADDTREE_OK) return st;
    if (a->B > 0 && a->ctx_len == nullptr) return fail(CADDTREE_E_INVALID, "ctx_len is NULL");
  }
  // The kernels form pos_i - window + 1 - pos_j in 32 bits, with a window below the sequence's length (args_of): from -T on
  // for the first position of more queries than keys, and for the new keys of a cache in their own numbers.
  const int64_t far = cache ? (int64_t)a->table_pages * CADDTREE_PAGE + 2 * (int64_t)a->T : a->T + 2 * (int64_t)a->S;
  if (a->window > 0 && far > (int64_t)1 << 31)
    return fail(CADDTREE_E_UNSUPPORTED, "a window over more than 2^31 positions: T + 2 S, or the table's slots + 2 T");
  return check_view("q", a->q, a->B > 0 && a->T > 0);
}

AttnArgs args_of(const caddtree_attention_t* a, const caddtree_cache_t* cache) {
  AttnArgs k = {};
  k.q = view(a->q);
  k.k = view(a->k);
  k.v = view(a->v);
  k.out = view(a->out);
  k.lse = a->lse;
  k.q_len = a->q_len;
  k.k_len = cache ? nullptr : a->k_len;
  k.B = a->B;
  k.T = a->T;
  k.S = a->S;
  k.Hq = a->n_heads;
  k.Hkv = a->n_kv_heads;
  k.G = a->n_heads / a->n_kv_heads;
  k.scale = a->scale;
  // All positions are below `reach`: a window that long hides no key and is none.
  const int64_t reach = cache ? (int64_t)a->table_pages * CADDTREE_PAGE + a->T : a->S;
  k.window = a->window >= reach ? 0 : a->window;
  k.sinks = a->sinks;
  k.order = enum_value(a->order);
  k.mask_kind = enum_value(a->mask_kind);
  k.mask = a->mask;
  k.depth = a->depth;
  k.cap = a->cap;
  if (cache) {
    k.kv = paged(cache, a->page_table, a->table_pages);
    k.ctx_len = a->ctx_len;
  }
  return k;
}

caddtree_status_t check_workspace(const void* workspace) {
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(CADDTREE_E_WORKSPACE, "workspace must be 256-byte aligned");
  return CADDTREE_OK;
}

// An array of a call and whether the call writes it.  What is written must lie in no other array: the kernels of a call
// read and write in no fixed order.
struct Array {
  const char* name;
  const void* data;
  size_t bytes;              // (of sizes within the limits: below 2^64)
  bool written;
};
template <size_t n>
caddtree_status_t check_apart(const Array (&all)[n]) {
  for (size_t i = 0; i < n; ++i)
    for (size_t j = i + 1; j < n; ++j) {
      const Array &x = all[i], &y = all[j];
      const uintptr_t px = reinterpret_cast<uintptr_t>(x.data), py = reinterpret_cast<uintptr_t>(y.data);
      if ((x.written || y.written) && x.bytes > 0 && y.bytes > 0 && (px <= py ? py - px < x.bytes : px - py < y.bytes))
        return fail(CADDTREE_E_INVALID, "%s and %s overlap", x.name, y.name);
    }
  return CADDTREE_OK;
}

// How many parts a row's keys are cut into, from the sizes alone (lengths are on the device): as many as fill the
// card, two workgroups a compute unit, where each keeps a few tiles: 192 keys for up to 64 rows (one token over 1024:
// 14.2 us, 15.8 with 384 keys), 384 for more, whose parts' sums are larger (65 rows of 4 heads over 4096: 25 us, 29.5
// with 192).  A call that fills the card by itself is not cut: the sums cost more than an uneven last round does (32
// trees of 257 rows, 2304 workgroups: 2% more in two parts).
int32_t splits_of(const caddtree_attention_t* a) {
  const int64_t G = a->n_heads / a->n_kv_heads, rows = a->T * G;
  const int64_t groups = (int64_t)a->B * a->n_kv_heads * (rows <= 64 ? 1 : (rows + 127) / 128);
  int64_t reach = (int64_t)a->table_pages * CADDTREE_PAGE + a->S;      // keys of a workgroup's rows at most
  if (a->window > 0) reach = std::min(reach, (int64_t)a->window + a->sinks + std::min<int64_t>(a->T, 128 / G + 1) + 64);
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(kResident / std::max<int64_t>(groups, 1), reach / (rows <= 64 ? 192 : 384)));
}
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t split_bytes(const caddtree_attention_t* a, int32_t n) {
  if (n <= 1) return 0;
  const size_t rows = (size_t)a->B * a->T * a->n_heads * n;
  return align256(rows * 8) + rows * a->head_dim * 4;
}

caddtree_status_t run_attention(const caddtree_attention_t* a, const caddtree_cache_t* cache, void* workspace, size_t bytes,
                                hipStream_t stream) {
  if (a->lse != nullptr && a->lse_strided) return fail(CADDTREE_E_INVALID, "lse is written contiguous: lse_strided must be 0");
  if (a->B == 0 || a->T == 0) return ok();
  caddtree::Split sp = {1, nullptr, nullptr};
  if (workspace != nullptr) {
    int32_t n = splits_of(a);
    while (n > 1 && split_bytes(a, n) > bytes) n /= 2;
    sp.n = n;
    sp.ml = static_cast<float*>(workspace);
    sp.sum = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256((size_t)a->B * a->T * a->n_heads * n * 8));
  }
  const hipError_t e = caddtree::launch_attention(args_of(a, cache), sp, (caddtree_dtype_t)enum_value(a->dtype), a->head_dim, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "attention launch");
}

}  // namespace

extern "C" {

size_t caddtree_attention_workspace_bytes(const caddtree_attention_t* a) {
  if (check_sizes(a) != CADDTREE_OK || a->B == 0 || a->T == 0) return 0;
  if (a->table_pages < 0 || (int64_t)a->table_pages * CADDTREE_PAGE > kMaxTokens) return 0;
  return split_bytes(a, splits_of(a));
}

caddtree_status_t caddtree_window_attention(const caddtree_attention_t* a, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  caddtree_status_t st = check_attention(a, nullptr);
  if (st != CADDTREE_OK) return st;
  const bool some = a->B > 0 && a->T > 0;
  if ((st = check_view("k", a->k, some && a->S > 0)) != CADDTREE_OK) return st;
  if ((st = check_view("v", a->v, some && a->S > 0)) != CADDTREE_OK) return st;
  if ((st = check_view("out", a->out, some)) != CADDTREE_OK) return st;
  if ((st = check_workspace(workspace)) != CADDTREE_OK) return st;
  return run_attention(a, nullptr, workspace, workspace_bytes, stream);
}

caddtree_status_t caddtree_cache_attention(const caddtree_cache_t* cache, const caddtree_attention_t* a, void* workspace,
                                           size_t workspace_bytes, hipStream_t stream) {
  if (cache == nullptr) return fail(CADDTREE_E_INVALID, "cache is NULL");
  caddtree_status_t st = check_attention(a, cache);
  if (st != CADDTREE_OK) return st;
  if ((st = check_view("k", a->k, false)) != CADDTREE_OK) return st;
  if ((st = check_view("v", a->v, a->k.data != nullptr)) != CADDTREE_OK) return st;
  if (a->v.data != nullptr && a->k.data == nullptr) return fail(CADDTREE_E_INVALID, "v is given without k");
  if ((st = check_view("out", a->out, a->B > 0 && a->T > 0)) != CADDTREE_OK) return st;
  if (enum_value(a->order) == CADDTREE_ORDER_TREE && a->k.data != nullptr && a->T > 1 &&
      (a->mask == nullptr || enum_value(a->mask_kind) == CADDTREE_MASK_NONE))
    return fail(CADDTREE_E_INVALID, "a tree's new keys need its mask");
  if ((st = check_workspace(workspace)) != CADDTREE_OK) return st;
  return run_attention(a, cache, workspace, workspace_bytes, stream);
}

caddtree_status_t caddtree_cache_write(const caddtree_cache_t* cache, const caddtree_view_t* k, const caddtree_view_t* v,
                                       int32_t B, int32_t T, int32_t rows, const int64_t* start, const int32_t* count,
                                       const int32_t* index, const int32_t* page_table, int32_t table_pages,
                                       hipStream_t stream) {
  caddtree_status_t st = check_cache(cache);
  if (st != CADDTREE_OK) return st;
  if ((st = check_batch(B)) != CADDTREE_OK) return st;
  if (T < 0 || rows < 0) return fail(CADDTREE_E_INVALID, "T = %d and rows = %d must not be negative", T, rows);
  if ((int64_t)T * cache->n_kv_heads > kMaxTokens)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d tokens of %d heads exceed 2^30", T, cache->n_kv_heads);
  if (index == nullptr && rows < T) return fail(CADDTREE_E_INVALID, "rows = %d hold fewer than T = %d tokens", rows, T);
  if (k == nullptr || v == nullptr) return fail(CADDTREE_E_INVALID, "k and v are required");
  if ((st = check_table("page_table", page_table, table_pages)) != CADDTREE_OK) return st;
  const bool some = B > 0 && T > 0 && table_pages > 0;
  if ((st = check_view("k", *k, some)) != CADDTREE_OK) return st;
  if ((st = check_view("v", *v, some)) != CADDTREE_OK) return st;
  if (B > 0 && start == nullptr) return fail(CADDTREE_E_INVALID, "start is NULL");
  if (!some) return ok();
  caddtree::CacheMoveArgs a = {view(*k), view(*v), paged(cache, page_table, table_pages), start, nullptr, count, index, B, T, rows};
  const hipError_t e = caddtree::launch_cache_write(a, (caddtree_dtype_t)enum_value(cache->dtype), cache->head_dim, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cache write launch");
}

caddtree_status_t caddtree_cache_read(const caddtree_cache_t* cache, const caddtree_view_t* k, const caddtree_view_t* v,
                                      int32_t B, int32_t T, const int64_t* start, const int64_t* end,
                                      const int32_t* page_table, int32_t table_pages, hipStream_t stream) {
  caddtree_status_t st = check_cache(cache);
  if (st != CADDTREE_OK) return st;
  if ((st = check_batch(B)) != CADDTREE_OK) return st;
  if (T < 0) return fail(CADDTREE_E_INVALID, "T = %d must not be negative", T);
  if ((int64_t)T * cache->n_kv_heads > kMaxTokens)
    return fail(CADDTREE_E_UNSUPPORTED, "T = %d tokens of %d heads exceed 2^30", T, cache->n_kv_heads);
  if (k == nullptr || v == nullptr) return fail(CADDTREE_E_INVALID, "k and v are required");
  if ((st = check_table("page_table", page_table, table_pages)) != CADDTREE_OK) return st;
  const bool some = B > 0 && T > 0 && table_pages > 0;
  if ((st = check_view("k", *k, some)) != CADDTREE_OK) return st;
  if ((st = check_view("v", *v, some)) != CADDTREE_OK) return st;
  if (B > 0 && end == nullptr) return fail(CADDTREE_E_INVALID, "end is NULL");
  if (!some) return ok();
  if (k->data == v->data) return fail(CADDTREE_E_INVALID, "k and v are written, and both begin in one place");
  caddtree::CacheMoveArgs a = {view(*k), view(*v), paged(cache, page_table, table_pages), start, end, nullptr, nullptr, B, T, T};
  const hipError_t e = caddtree::launch_cache_read(a, (caddtree_dtype_t)enum_value(cache->dtype), cache->head_dim, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cache read launch");
}

caddtree_status_t caddtree_cache_score(const caddtree_cache_t* cache, const caddtree_attention_t* a, const float* weight,
                                       const float* scores, float* new_scores, int64_t slots, hipStream_t stream) {
  if (cache == nullptr) return fail(CADDTREE_E_INVALID, "cache is NULL");
  caddtree_status_t st = check_attention(a, cache);
  if (st != CADDTREE_OK) return st;
  if (slots < 0 || slots > kMaxTokens) return fail(CADDTREE_E_INVALID, "slots = %lld must be in 0 .. 2^30", (long long)slots);
  if (a->B == 0 || slots == 0) return ok();
  if (a->T > 0 && a->lse == nullptr) return fail(CADDTREE_E_INVALID, "lse is NULL");
  if (a->lse_strided && (a->lse_stride_b < 0 || a->lse_stride_t < 0 || a->lse_stride_h < 0))
    return fail(CADDTREE_E_INVALID, "the strides of lse must not be negative");
  if (scores == nullptr || new_scores == nullptr) return fail(CADDTREE_E_INVALID, "scores and new_scores are required");
  if (new_scores != scores) {
    const size_t bytes = (size_t)a->B * a->n_kv_heads * slots * 4;
    const Array arrays[] = {{"scores", scores, bytes, false}, {"new_scores", new_scores, bytes, true}};
    if ((st = check_apart(arrays)) != CADDTREE_OK) return st;
  }
  caddtree::ScoreArgs s = {args_of(a, cache), weight, scores, new_scores, slots, (int64_t)a->T * a->n_heads, a->n_heads, 1};
  if (a->lse_strided) {
    s.lse_b = a->lse_stride_b;
    s.lse_t = a->lse_stride_t;
    s.lse_h = a->lse_stride_h;
  }
  const hipError_t e = caddtree::launch_cache_score(s, (caddtree_dtype_t)enum_value(a->dtype), a->head_dim, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cache score launch");
}

size_t caddtree_evict_workspace_bytes(const caddtree_cache_t* cache, int32_t B, int32_t table_pages, int64_t slots) {
  if (check_cache(cache) != CADDTREE_OK || check_batch(B) != CADDTREE_OK || table_pages < 0 || slots < 0 || slots > kMaxTokens) return 0;
  return caddtree::evict_workspace_bytes(paged(cache, nullptr, table_pages), B, slots);
}

caddtree_status_t caddtree_cache_evict(const caddtree_cache_t* cache, int32_t B, const int32_t* page_table,
                                       int32_t table_pages, const int64_t* ctx_len, const float* scores, int64_t slots,
                                       int32_t budget, int32_t sinks, int32_t recent, const int32_t* new_table,
                                       int32_t new_pages, float* new_scores, int64_t new_slots, int64_t* new_len,
                                       int32_t* kept, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  caddtree_status_t st = check_cache(cache);
  if (st != CADDTREE_OK) return st;
  if ((st = check_batch(B)) != CADDTREE_OK) return st;
  if ((st = check_table("page_table", page_table, table_pages)) != CADDTREE_OK) return st;
  if ((st = check_table("new_table", new_table, new_pages)) != CADDTREE_OK) return st;
  if (budget < 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return fail(CADDTREE_E_INVALID, "sinks = %d and recent = %d must not be negative and must fit budget = %d", sinks, recent, budget);
  if (slots < 0 || slots > kMaxTokens || new_slots < budget || new_slots > kMaxTokens)
    return fail(CADDTREE_E_INVALID, "slots = %lld must be in 0 .. 2^30 and new_slots = %lld in budget = %d .. 2^30",
                (long long)slots, (long long)new_slots, budget);
  if ((int64_t)new_pages * CADDTREE_PAGE < budget)
    return fail(CADDTREE_E_INVALID, "new_table's %d pages hold fewer than budget = %d slots", new_pages, budget);
  if (B == 0) return ok();
  if (ctx_len == nullptr || new_len == nullptr) return fail(CADDTREE_E_INVALID, "ctx_len and new_len are required");
  if ((slots > 0 && scores == nullptr) || (new_slots > 0 && new_scores == nullptr) || (budget > 0 && kept == nullptr))
    return fail(CADDTREE_E_INVALID, "scores, new_scores and kept are required");
  if ((st = check_workspace(workspace)) != CADDTREE_OK) return st;
  const size_t bytes = caddtree::evict_workspace_bytes(paged(cache, page_table, table_pages), B, slots);
  if (bytes > 0 && (workspace == nullptr || workspace_bytes < bytes))
    return fail(CADDTREE_E_WORKSPACE, "rows of %lld slots need a workspace of %zu bytes, got %zu", (long long)slots, bytes,
                workspace ? workspace_bytes : (size_t)0);
  const size_t rows = (size_t)B * cache->n_kv_heads;
  const Array arrays[] = {{"page_table", page_table, (size_t)B * table_pages * 4, false},
                          {"ctx_len", ctx_len, (size_t)B * 8, false},
                          {"scores", scores, rows * slots * 4, false},
                          {"new_table", new_table, (size_t)B * new_pages * 4, false},
                          {"new_scores", new_scores, rows * new_slots * 4, true},
                          {"new_len", new_len, (size_t)B * 8, true},
                          {"kept", kept, rows * budget * 4, true},
                          {"workspace", workspace, bytes, true},
                          {"the cache's pages", cache->pages,
                           (size_t)(cache->n_pages * cache->n_kv_heads * CADDTREE_PAGE_BYTES(cache->head_dim)), true}};
  if ((st = check_apart(arrays)) != CADDTREE_OK) return st;
  if (new_table == page_table && budget > 0)
    return fail(CADDTREE_E_INVALID, "new_table is page_table: kept slots go to pages that are not in use");
  caddtree::EvictArgs a = {paged(cache, page_table, table_pages), B, cache->head_dim, ctx_len, scores, slots, budget, sinks,
                           recent, new_table, new_pages, new_scores, new_slots, new_len, kept};
  const hipError_t e = caddtree::launch_cache_evict(a, workspace, stream);
  return e == hipSuccess ? ok() : hip_fail(e, "cache evict launch");
}

}  // extern "C"
