// Arguments of the attention and cache kernels, filled by attention_api.cpp.  Host-only sources include
// it, so it declares no device code.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "caddtree.h"

namespace caddtree {

struct View {                // [B, tokens, heads, head_dim], strides in elements
  char* data;
  int64_t b, t, h;
};

struct PagedKV {
  uint8_t* pages;            // null: no cache
  int64_t n_pages;
  const int32_t* table;      // [B, table_pages]
  int32_t table_pages;
  int32_t heads;             // kv heads of a page
  int32_t page_bytes;        // of one page and head
};

struct AttnArgs {
  View q, k, v, out;         // k.data null: no new keys
  float* lse;                // [B, T, Hq] or null
  const int32_t* q_len;      // [B] or null
  const int32_t* k_len;      // [B] or null
  int32_t B, T, S, Hq, Hkv, G;
  float scale;
  int32_t window, sinks;
  int32_t order;             // caddtree_order_t
  int32_t mask_kind;         // caddtree_mask_t of a tree
  const void* mask;
  const int32_t* depth;      // [B, cap] of a tree (order says whether the queries are one's)
  int32_t cap;
  PagedKV kv;
  const int64_t* ctx_len;    // [B]
};

// The tiles of a row in n parts, each a workgroup's; above 1 their results go to the workspace.
struct Split {
  int32_t n;
  float* ml;                 // [B, Hkv, T G, n, 2]
  float* sum;                // [B, Hkv, T G, n, head_dim]
};
hipError_t launch_attention(const AttnArgs& a, const Split& sp, caddtree_dtype_t dtype, int32_t head_dim, hipStream_t stream);

struct CacheMoveArgs {       // write: views -> slots; read: slots -> views
  View k, v;
  PagedKV kv;
  const int64_t* start;      // [B] or null (0)
  const int64_t* end;        // read: [B]
  const int32_t* count;      // write: [B] or null (T)
  const int32_t* index;      // write: [B, T] or null
  int32_t B, T, rows;
};
hipError_t launch_cache_write(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t head_dim, hipStream_t stream);
hipError_t launch_cache_read(const CacheMoveArgs& a, caddtree_dtype_t dtype, int32_t head_dim, hipStream_t stream);

struct ScoreArgs {
  AttnArgs at;               // q, lse, lengths, visibility and the cache
  const float* weight;       // [B, T] or null
  const float* scores;       // [B, Hkv, slots]
  float* new_scores;
  int64_t slots;
  int64_t lse_b, lse_t, lse_h;   // strides of at.lse
};
hipError_t launch_cache_score(const ScoreArgs& a, caddtree_dtype_t dtype, int32_t head_dim, hipStream_t stream);

struct EvictArgs {
  PagedKV kv;
  int32_t B, head_dim;
  const int64_t* ctx_len;
  const float* scores;       // [B, heads, slots]
  int64_t slots;
  int32_t budget, sinks, recent;
  const int32_t* new_table;  // [B, new_pages]
  int32_t new_pages;
  float* new_scores;         // [B, heads, new_slots]
  int64_t new_slots;
  int64_t* new_len;          // [B]
  int32_t* kept;             // [B, heads, budget]
};
size_t evict_workspace_bytes(const PagedKV& kv, int32_t B, int64_t slots);
hipError_t launch_cache_evict(const EvictArgs& a, void* workspace, hipStream_t stream);

}  // namespace caddtree
