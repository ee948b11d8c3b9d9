// Attention over the keys of a tensor and of a 4-bit cache, in three kernels by the rows (queries x heads) that
// share a kv head.  All go over the keys once with the running maximum and sum of a softmax, and form S^T = K Q^T and
// O^T = V^T P^T, so that a row's statistics and sums lie in lanes of the row.
//
// Over a cache few rows (at most 32: single tokens, small blocks) are bound by reading the keys.  The narrow kernel's
// wavefronts each take tiles of their own: codes go from memory to registers, keys are converted there into the
// operand of the matrix product, values pass through LDS to be transposed.  33 to 64 rows would convert a tile more
// often than it is used; the pair kernel's four wavefronts share it.  Many rows (prompts, trees) are bound by the
// matrix products and the softmax; the wide kernel's four wavefronts share each tile and hold 32 rows each.
// Over 131072 cached keys of 8 kv heads: 32 rows narrow 48 us, pair 66; 64 rows pair 69, wide 82.
//
// A tensor's tiles go to LDS by themselves, so the wide kernel takes few rows as well: over 131072 keys 4 rows 49 us,
// narrow 58; 32 rows 56 us, narrow 69; 64 rows 73 us, pair 82.  Where there are few keys in all (kFewKeys) and up to 16
// rows the narrow kernel starts and ends sooner: 1000 keys of 8 kv heads 9.9 us, wide 11.9; 1028 of 64 14.3 us, wide
// 14.9; 1024 of 512 28.5 us, wide 22.9.
//
// Where there are too few workgroups for the card, the tiles of a row are split over several, whose
// partial sums the combining kernel joins in a fixed order.
#include <algorithm>

#include "attn_tile.h"

namespace caddtree {
namespace {

using namespace at;

constexpr int64_t kFewKeys = 1 << 17;               // of all sequences and kv heads
constexpr int kMaxSplits = 512, kFewSplits = 8;      // (attention_api.cpp: at most as many as workgroups fill the card)

// partial results of (sequence, kv head, row, split): D sums, relative to the maximum, in `sum`; the
// maximum (in units of log2) and the sum of the weights in `ml`
__device__ int64_t part_of(const AttnArgs& a, const Split& sp, int b, int hk, int r) {
  return (((int64_t)b * a.Hkv + hk) * ((int64_t)a.T * a.G) + r) * sp.n;
}

// ---------------------------------------------------------------- few rows

// A wavefront's tile of a page: lane (col, g) holds the codes of tokens 16 s + col, channels g D / 4 .. of
// keys, and whole blocks of values, token by token.
template <int D>
struct PageStage {
  uint32_t kc[4][D / 32] = {};
  uint32_t ks[4] = {};
  u32x4 vc[D / 32] = {};
  uint32_t vs[D / 32] = {};

  __device__ void load_keys(const uint8_t* page, int lane) {
    using L = PageLayout<D>;
    const uint32_t col = lane & 15, g = lane >> 4;
    if (page == nullptr) return;                    // (no key of it is seen: what the registers hold does not matter)
    const uint32_t code = col * L::kRow + g * (D / 8), scale = col * L::kScales + g * (D / 4) / kBlock;
    const uint8_t* scales = page + L::kKs;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint32_t* c = reinterpret_cast<const uint32_t*>(page + (code + 16 * s * L::kRow));
#pragma unroll
      for (int w = 0; w < D / 32; ++w) kc[s][w] = c[w];
      ks[s] = scales[scale + 16 * s * L::kScales];
    }
  }
  __device__ void load_values(const uint8_t* page, int lane) {
    using L = PageLayout<D>;
    if (page == nullptr) return;
    const uint8_t *codes = page + L::kV, *scales = page + L::kVs;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      vc[u] = *reinterpret_cast<const u32x4*>(codes + ((uint32_t)lane * 16 + u * 1024));
      vs[u] = scales[(uint32_t)lane + 64 * u];
    }
  }
  // the operand of keys 16 s .. 16 s + 15: D / 32 instructions' worth
  template <typename E>
  __device__ void keys(int s, u32x4 out[D / 32]) const {
    const float f = scale_of(ks[s]);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      out[j][0] = E::template from4<0>(kc[s][j], f);
      out[j][1] = E::template from4<1>(kc[s][j], f);
      out[j][2] = E::template from4<2>(kc[s][j], f);
      out[j][3] = E::template from4<3>(kc[s][j], f);
    }
    if (ks[s] == 255) out[0][0] = E::kNaN;          // (one is enough for the key's scores)
  }
  // values of tokens 32 half .. + 31 into LDS.  there: tokens of the tile that are there; returns whether a
  // tile that is not seen in full had any that are not finite
  template <typename E>
  __device__ bool values(int half, char* lds, int lane, bool full, int there) const {
    constexpr int kPer = D / 32, kU = kPer / 2;    // blocks of a token; loads of a half
    bool odd = false;
#pragma unroll
    for (int v = 0; v < kU; ++v) {
      const int u = half * kU + v, q = lane + 64 * u, token = q / kPer, blk = q % kPer, row = token & 31;
      uint32_t x[16];
      decode_block<E>(vc[u], vs[u], x);
      if (!full) {
        const bool gone = token >= there, nan = !gone && vs[u] == 255;
        if (gone || nan)
#pragma unroll
          for (int w = 0; w < 16; ++w) x[w] = 0;
        odd = odd || nan;
      }
#pragma unroll
      for (int w = 0; w < 4; ++w)
        *reinterpret_cast<u32x4*>(lds + v_at<D>(row, blk * 64 + w * 16)) =
            u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
    }
    return odd;
  }
};

// A wavefront's tile of 32 keys of a tensor.
template <int D>
struct TensorStage {
  u32x4 kr[2][D / 32];
  u32x4 vr[D / 16];

  __device__ void load_keys(const char* k, int64_t kt, int j0, int nk, int lane) {
    const int col = lane & 15, g = lane >> 4;
    const char* base = k + 2 * (j0 * kt);           // (uniform; a lane's offset in a tile is below 2^32: see kMaxStride)
#pragma unroll
    for (int s = 0; s < 2; ++s) {                   // (a key that is not there: the tile's first one in its place)
      const uint32_t row = j0 + 16 * s + col < nk ? 16 * s + col : 0;
      const u32x4* p = reinterpret_cast<const u32x4*>(base + (row * (2 * (uint32_t)kt) + (uint32_t)g * (D / 2)));
#pragma unroll
      for (int j = 0; j < D / 32; ++j) kr[s][j] = p[j];
    }
  }
  __device__ void load_values(const char* v, int64_t vt, int j0, int nk, int lane) {
    const char* base = v + 2 * (j0 * vt);
    const uint32_t piece = lane % (D / 8) * 16;
#pragma unroll
    for (int u = 0; u < D / 16; ++u) {
      const int token = lane / (D / 8) + u * (512 / D);
      vr[u] = *reinterpret_cast<const u32x4*>(base + ((uint32_t)(j0 + token < nk ? token : 0) * (2 * (uint32_t)vt) + piece));
    }
  }
  template <typename E>
  __device__ void keys(int s, u32x4 out[D / 32]) const {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) out[j] = kr[s][j];
  }
  template <typename E>
  __device__ bool values(int, char* lds, int lane, bool full, int there) const {
    bool odd = false;
#pragma unroll
    for (int u = 0; u < D / 16; ++u) {
      const int token = lane / (D / 8) + u * (512 / D);
      u32x4 x = vr[u];
      if (!full) {
        if (token >= there) x = u32x4{0, 0, 0, 0};
        if (clean_pairs<E>(x)) odd = true;
      }
      *reinterpret_cast<u32x4*>(lds + v_at<D>(token, lane % (D / 8) * 16)) = x;
    }
    return odd;
  }
};

// The running softmax of 16 kR rows: lane (col, g) has rows 16 n + col and channels 16 t + 4 g .. + 3.
template <int D, int kR>
struct NarrowState {
  float m[kR], l[kR];
  f32x4 acc[D / 16][kR];
};

// Takes a tile of 32 kH keys.  next_keys, next_values: load the following tile's into the registers that this
// one's have left.  Returns whether a lane met values that are not finite in a tile not seen in full.
template <typename E, int D, int kR, int kH, typename Stage, typename NextKeys, typename NextValues>
__device__ __forceinline__ bool narrow_tile(NarrowState<D, kR>& st, Stage& x, const u32x4 (&q)[kR][D / 32], float c, bool full,
                            const uint64_t (&seen)[kR], int there, char* lds, int lane, NextKeys next_keys,
                            NextValues next_values) {
  const int g = lane >> 4;
  bool odd = false;
  f32x4 s[2 * kH][kR];
#pragma unroll
  for (int t = 0; t < 2 * kH; ++t) {
    u32x4 k[D / 32];
    x.template keys<E>(t, k);
#pragma unroll
    for (int n = 0; n < kR; ++n) {
      s[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) s[t][n] = Mfma<E>::m16(k[j], q[n][j], s[t][n]);
    }
  }
  next_keys();
  u32x4 p[kH][kR];
#pragma unroll
  for (int n = 0; n < kR; ++n) {
    float top = -INFINITY;
    const uint64_t bits = seen[n] >> (4 * g);       // key 16 t + 4 g + r is bit 16 t + r
#pragma unroll
    for (int t = 0; t < 2 * kH; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (!full && !((bits >> (16 * t + r)) & 1)) s[t][n][r] = -INFINITY;
        top = fmaxf(top, s[t][n][r]);
      }
    top = max_across_32(max_across_16(top)) * c;
    if (__any(top > st.m[n] + kLag)) {
      const float m = fmaxf(st.m[n], top), was = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[n] - m);
      st.l[n] *= was;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) st.acc[t][n] *= was;
      st.m[n] = m;
    }
    const float base = st.m[n] == -INFINITY ? 0.f : st.m[n] - E::kBias;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2 * kH; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][n][r], c, -base));
        sum += s[t][n][r];
      }
    st.l[n] += sum;                                 // (of this lane's keys: the four g are added at the end)
#pragma unroll
    for (int h = 0; h < kH; ++h)
      p[h][n] = u32x4{E::pair(s[2 * h][n][0], s[2 * h][n][1]), E::pair(s[2 * h][n][2], s[2 * h][n][3]),
                      E::pair(s[2 * h + 1][n][0], s[2 * h + 1][n][1]), E::pair(s[2 * h + 1][n][2], s[2 * h + 1][n][3])};
  }
#pragma unroll
  for (int h = 0; h < kH; ++h) {
    __builtin_amdgcn_wave_barrier();
    if (x.template values<E>(h, lds, lane, full, there)) odd = true;
    if (h == kH - 1) next_values();
    __builtin_amdgcn_wave_barrier();
    const int v0 = v_at<D>(4 * g + (lane & 15) / 4, (lane & 3) * 8);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {              // (16 rows further: the same swizzle)
      const char* at = lds + (v0 ^ v_step(32 * t));
      const u32x2 lo = read_transposed(at), hi = read_transposed(at + 16 * 2 * D);
      const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
      for (int n = 0; n < kR; ++n) st.acc[t][n] = Mfma<E>::m16(v, p[h][n], st.acc[t][n]);
    }
  }
  return odd;
}

// Up to 16 kR rows.  Bound by reading the keys: 64 single tokens over 4096 to 8192 cached ones, 8 kv heads of 128
// channels, take 92 us, 5.0 TB/s of codes and scales: what a large copy reaches on this card, 71% of a pure read.  A wavefront has a page's
// codes on their way while it takes the page before (a page is 8.5 KB, eight wavefronts a compute unit), and the next
// pages' numbers before that: a number waited for in the loop would hold up the loads behind it.
template <typename E, int D, int kR, bool kPaged>
__global__ __launch_bounds__(256, 2) void narrow_kernel(AttnArgs a, Split sp) {
  using L = PageLayout<D>;
  constexpr int kVBytes = 32 * 2 * D;               // 32 tokens' values; as many fp32 sums of 16 rows
  __shared__ __align__(16) char lds[4 * kVBytes];
  __shared__ float ml[4][2][16 * kR];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.G;
  if (R == 0) return;
  const Span span = span_of<kPage, 32>(a, s, 0, s.nq - 1);
  const int per = ceil_div(span.n, sp.n), t0 = split * per, t1 = min(span.n, t0 + per);

  u32x4 q[kR][D / 32];
  RowAt rows[kR];
#pragma unroll
  for (int n = 0; n < kR; ++n) {
    const int r = min(16 * n + col, R - 1), i = r / a.G, h = hk * a.G + r % a.G;
    rows[n] = row_at(a, s, b, i);
    const u32x4* p = reinterpret_cast<const u32x4*>(a.q.data + 2 * (b * a.q.b + i * a.q.t + h * a.q.h + g * (D / 4)));
#pragma unroll
    for (int j = 0; j < D / 32; ++j) q[n][j] = signed_queries(p[j], a.scale);
  }
  NarrowState<D, kR> st;
#pragma unroll
  for (int n = 0; n < kR; ++n) {
    st.m[n] = -INFINITY;
    st.l[n] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) st.acc[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c = score_factor(a.scale);
  char* vt = lds + wave * kVBytes;
  uint64_t seen[kR];
  bool odd = false;
  const char* kb = a.k.data + 2 * (b * a.k.b + hk * a.k.h);
  const char* vb = a.v.data + 2 * (b * a.v.b + hk * a.v.h);
  auto sees = [&](bool cached, const RowAt& row, int at) -> uint64_t {
    if (kPaged && cached) return sees_cached(a, s, row).at(at);
    if (kPaged && a.order == CADDTREE_ORDER_TREE) return sees_tree(a, s, b, row, at);
    return sees_new(a, s, row).at(at);
  };

  int t = t0 + wave;
  if constexpr (kPaged) {
    const int nc = min(t1, span.a + span.c - span.b);    // this split's cached tiles come first
    PageStage<D> x;
    auto entry = [&](int tile) -> int32_t {
      bool cached;
      return tile < nc ? table_entry(a.kv, b, tile_of<kPage, 32>(span, tile, &cached) / kPage) : -1;
    };
    const uint8_t* page = page_at(a.kv, entry(t), hk);
    int32_t ahead = entry(t + 4);
    x.load_keys(page, lane);
    x.load_values(page, lane);
    for (; t < nc; t += 4) {
      bool cached;
      const int at = tile_of<kPage, 32>(span, t, &cached);
      const int32_t after = entry(t + 8);
      const uint8_t* next = nullptr;
      const bool full = page && full_cached(a, s, s.nq - 1, at, kPage);
#pragma unroll
      for (int n = 0; n < kR; ++n) seen[n] = full ? ~0ull : page ? sees(true, rows[n], at) : 0;
      if (narrow_tile<E, D, kR, 2>(
              st, x, q, c, full, seen, page ? s.ctx - at : 0, vt, lane,
              [&] {
                next = page_at(a.kv, ahead, hk);
                x.load_keys(next, lane);
              },
              [&] { x.load_values(next, lane); }))
        odd = true;
      page = next;
      ahead = after;
    }
  }
  {
    // A cache's few new tiles (kPaged) are loaded as they are needed: keys, then values while the weights are
    // formed, which keeps the registers of this loop below those of the cached one's.
    TensorStage<D> x;
    bool cached;
    int at = t < t1 ? tile_of<kPage, 32>(span, t, &cached) : 0;
    if (!kPaged && t < t1) {
      x.load_keys(kb, a.k.t, at, s.nk, lane);
      x.load_values(vb, a.v.t, at, s.nk, lane);
    }
    for (; t < t1; t += 4) {
      const bool more = t + 4 < t1;
      const int after = more ? tile_of<kPage, 32>(span, t + 4, &cached) : 0;
      const bool full = full_new(a, s, 0, s.nq - 1, at, 32);
#pragma unroll
      for (int n = 0; n < kR; ++n) seen[n] = full ? ~0ull : sees(false, rows[n], at);
      if (kPaged) x.load_keys(kb, a.k.t, at, s.nk, lane);
      if (narrow_tile<E, D, kR, 1>(
              st, x, q, c, full, seen, s.nk - at, vt, lane,
              [&] {
                if (kPaged) x.load_values(vb, a.v.t, at, s.nk, lane);
                else if (more) x.load_keys(kb, a.k.t, after, s.nk, lane);
              },
              [&] { if (!kPaged && more) x.load_values(vb, a.v.t, after, s.nk, lane); }))
        odd = true;
      at = after;
    }
  }
  if (__any(odd)) {
    for (t = t0 + wave; t < t1; t += 4) {
      bool cached;
      const int at = tile_of<kPage, 32>(span, t, &cached), n = min(cached ? 64 : 32, (cached ? s.ctx : s.nk) - at);
      const uint8_t* page = kPaged && cached ? page_of(a.kv, b, at / kPage, hk) : nullptr;
      if (cached ? page == nullptr || full_cached(a, s, s.nq - 1, at, kPage) : full_new(a, s, 0, s.nq - 1, at, 32)) continue;
#pragma unroll
      for (int r = 0; r < kR; ++r) seen[r] = sees(cached, rows[r], at);
      for (int token = 0; token < n; ++token) {
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
          f32x4 v;
          if (kPaged && cached) {
            const float x = page[L::kVs + token * L::kScales + 16 * u / kBlock] == 255 ? __builtin_nanf("") : 0.f;
            v = f32x4{x, x, x, x};
          } else {
            v = unclean<E>(vb + 2 * ((at + token) * a.v.t + 16 * u + 4 * g));
          }
#pragma unroll
          for (int r = 0; r < kR; ++r)
            if ((seen[r] >> token) & 1) st.acc[u][r] += v;
        }
      }
    }
  }

  // the four wavefronts' sums, 16 rows at a time: a thread adds D / 16 channels of a row
#pragma unroll
  for (int n = 0; n < kR; ++n) {
    st.l[n] += __shfl_xor(st.l[n], 16);
    st.l[n] += __shfl_xor(st.l[n], 32);
    if (g == 0) {
      ml[wave][0][16 * n + col] = st.m[n];
      ml[wave][1][16 * n + col] = st.l[n];
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kR; ++n) {
    float m = -INFINITY;
    for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w][0][16 * n + col]);
    const float f = st.m[n] == -INFINITY ? (st.l[n] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(st.m[n] - m);
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
      *reinterpret_cast<f32x4*>(vt + col * (4 * D) + (((4 * t + g) ^ (col & 7)) << 4)) = st.acc[t][n] * f;
    __syncthreads();
    const int row = tid >> 4, part = tid & 15, r = 16 * n + row;
    if (r < R) {
      float mm = -INFINITY, ll = 0.f;
      for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[w][0][r]);
      for (int w = 0; w < 4; ++w) {
        const float mw = ml[w][0][r], lw = ml[w][1][r];
        ll += lw == 0.f ? 0.f : mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - mm);
      }
      f32x4 o[D / 64];
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < 4; ++w)
          if (ml[w][1][r] != 0.f)
            o[j] += *reinterpret_cast<const f32x4*>(lds + w * kVBytes + row * (4 * D) + (((part * (D / 64) + j) ^ (row & 7)) << 4));
      }
      const int i = r / a.G, h = hk * a.G + r % a.G, d = part * (D / 16);
      if (sp.n == 1) {
        const float inv = ll == 0.f ? 0.f : 1.f / ll;
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out.data + 2 * (b * a.out.b + i * a.out.t + h * a.out.h + d));
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          const u32x2 y = {E::pair(o[j][0] * inv, o[j][1] * inv), E::pair(o[j][2] * inv, o[j][3] * inv)};
          *reinterpret_cast<u32x2*>(dst + 2 * j) = y;
        }
        if (a.lse && part == 0)
          a.lse[((int64_t)b * a.T + i) * a.Hq + h] = ll == 0.f ? -INFINITY : (mm - E::kBias + __builtin_amdgcn_logf(ll)) * kLn2;
      } else {
        const int64_t at = part_of(a, sp, b, hk, r) + split;
        if (part == 0) {
          sp.ml[2 * at] = mm;
          sp.ml[2 * at + 1] = ll;
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j) *reinterpret_cast<f32x4*>(sp.sum + at * D + d + 4 * j) = o[j];
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- many rows

// A tile's 64 keys, or values, on their way to LDS: a share of a workgroup's 256 threads of a tensor's rows ...
template <int D>
struct TensorPart {
  static constexpr int kRows = 2048 / D, kN = 64 / kRows;      // rows a step (16 or 32); 16-byte pieces a thread
  u32x4 x[kN];
  __device__ void load(const char* p, int64_t stride, int j0, int nk, int tid) {
    const char* base = p + 2 * (j0 * stride);
    const uint32_t piece = k_piece<D>(tid % (D / 8)) * 16;
#pragma unroll
    for (int u = 0; u < kN; ++u) {                  // (a key that is not there: the tile's first one in its place)
      const int token = tid / (D / 8) + u * kRows;
      const uint32_t row = j0 + token < nk ? token : 0;
      x[u] = *reinterpret_cast<const u32x4*>(base + (row * (2 * (uint32_t)stride) + piece));
    }
  }
  // (kRows rows further: the same swizzle)
  __device__ void store_keys(char* lds, int tid) const {
    const int at = k_at<D>(tid / (D / 8), k_piece<D>(tid % (D / 8)));
#pragma unroll
    for (int u = 0; u < kN; ++u) *reinterpret_cast<u32x4*>(lds + at + u * kRows * 2 * D) = x[u];
  }
  template <typename E>
  __device__ void store_values(char* lds, int tid, bool full, int there, uint32_t* odd) {
    const int row = tid / (D / 8), at = v_at<D>(row, k_piece<D>(tid % (D / 8)) * 16);
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      if (!full) {
        if (row + u * kRows >= there) x[u] = u32x4{0, 0, 0, 0};
        if (clean_pairs<E>(x[u])) *odd = 1;
      }
      *reinterpret_cast<u32x4*>(lds + at + u * kRows * 2 * D) = x[u];
    }
  }
};
// A tile of keys or values straight to LDS: each lane fetches the 16 bytes that belong in its place of the tile, so
// nothing passes through registers.  The caller waits (tiles_there) before the barrier that hands the tile over.
template <int D>
struct TileMove {
  static constexpr int kRows = 2048 / D, kN = 64 / kRows;      // rows a step of the workgroup
  uint32_t from, to;         // a lane's bytes in a step's rows, the wavefront's place in a tile's step
  __device__ TileMove(int64_t stride, int tid, int wave, bool keys) {
    const int row = tid / (D / 8), n = tid % (D / 8);
    from = (uint32_t)row * (2 * (uint32_t)stride) + 16 * (keys ? k_there<D>(row, n) : v_there<D>(row, n));
    to = (uint32_t)wave * 1024;
  }
  __device__ __forceinline__ void send(const char* p, int64_t stride, int j0, uint32_t lds) const {
    const char* at = p + 2 * (j0 * stride);
    const int64_t step = 2 * kRows * stride;
    lds += to;
#pragma unroll
    for (int u = 0; u < kN; ++u, at += step, lds += 4096)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds), "v"(from), "s"(at) : "memory", "m0");
  }
};
__device__ __forceinline__ void tiles_there() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ... and of a page: a block of 32 channels of a key and one of a value a thread (D = 64: half of the threads)
template <int D>
struct PagePart {
  static constexpr int kBlocks = kPage * (D / kBlock);
  u32x4 k = {}, v = {};
  uint32_t ks = 0, vs = 0;
  __device__ void load(const uint8_t* page, int tid) {
    using L = PageLayout<D>;
    if (page == nullptr || tid >= kBlocks) return;  // (no key of a page that is not there is seen)
    const uint8_t *values = page + L::kV, *k_scales = page + L::kKs, *v_scales = page + L::kVs;
    k = *reinterpret_cast<const u32x4*>(page + (uint32_t)tid * 16);
    v = *reinterpret_cast<const u32x4*>(values + (uint32_t)tid * 16);
    ks = k_scales[(uint32_t)tid];
    vs = v_scales[(uint32_t)tid];
  }
  template <typename E>
  __device__ void store(char* keys, char* values, int tid, bool full, int there, uint32_t* odd) const {
    if (tid >= kBlocks) return;
    const int token = tid / (D / kBlock), blk = tid % (D / kBlock);
    uint32_t x[16];
    decode_block<E>(k, ks, x);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      *reinterpret_cast<u32x4*>(keys + k_at<D>(token, blk * 4 + w)) = u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
    decode_block<E>(v, vs, x);
    if (!full) {
      const bool gone = token >= there, nan = !gone && vs == 255;
      if (nan) *odd = 1;
      if (gone || nan)
#pragma unroll
        for (int w = 0; w < 16; ++w) x[w] = 0;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w)
      *reinterpret_cast<u32x4*>(values + v_at<D>(token, blk * 64 + w * 16)) = u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
  }
};

// A row's running softmax: lane (col, half) has row col and channels 32 d + 8 (e / 4) + 4 half + e % 4.
template <int D>
struct WideState {
  float m = -INFINITY, l = 0.f;
  f32x16 acc[D / 32];
};

// Scores of 32 kH keys: x[u] has row col's keys 32 u + 8 (e / 4) + 4 half + e % 4.  k0: the lane's first place in
// them.  The chains of products alternate, and their keys leave LDS three steps ahead.
template <typename E, int D, int kH>
__device__ __forceinline__ void wide_scores(f32x16 (&x)[kH], const u32x4 (&q)[D / 16], const char* keys, int k0) {
#pragma unroll
  for (int u = 0; u < kH; ++u)
#pragma unroll
    for (int e = 0; e < 16; ++e) x[u][e] = 0.f;
#pragma unroll
  for (int j = 0; j < D / 16; ++j)
#pragma unroll
    for (int u = 0; u < kH; ++u)
      x[u] = Mfma<E>::m32(*reinterpret_cast<const u32x4*>(keys + 64 * D * u + (k0 ^ k_step<D>(j))), q[j], x[u]);
  __builtin_amdgcn_sched_group_barrier(0x100, 3 * kH, 0);
#pragma unroll
  for (int j = 0; j < D / 16 - 3; ++j) {
    __builtin_amdgcn_sched_group_barrier(0x008, kH, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, kH, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 3 * kH, 0);
}
// ... of 32 kH keys: unseen ones left out and the row's maximum raised over them, where it lags too far behind.
// seen: bit k for the lane's key 32 u + 8 (e / 4) + e % 4.
template <typename E, int D, int kH>
__device__ __forceinline__ void wide_raise(WideState<D>& st, f32x16 (&x)[kH], float c, bool full, uint64_t seen) {
  if (!full) {
#pragma unroll
    for (int u = 0; u < kH; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[u][e] = (seen >> (32 * u + 8 * (e / 4) + e % 4)) & 1 ? x[u][e] : -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < kH; ++u)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, x[u][e]);
  top = max_across_32(top) * c;
  if (__any(top > st.m + kLag)) {
    const float m = fmaxf(st.m, top), was = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
    st.l *= was;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) st.acc[d] *= was;
    st.m = m;
  }
}
// weights of 32 keys, rounded to the inputs' type for the product with the values (their sum is not)
template <typename E, int D>
__device__ __forceinline__ void wide_weights(WideState<D>& st, f32x16& x, u32x4 (&p)[2], float c) {
  const float base = st.m == -INFINITY ? 0.f : st.m - E::kBias;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -base));
    st.l += x[e];                                   // (of this half's keys)
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
    p[u] = u32x4{E::pair(x[8 * u], x[8 * u + 1]), E::pair(x[8 * u + 2], x[8 * u + 3]), E::pair(x[8 * u + 4], x[8 * u + 5]),
                 E::pair(x[8 * u + 6], x[8 * u + 7])};
}
// ... times the values; v0: the lane's first place in them
template <typename E, int D>
__device__ __forceinline__ void wide_values(WideState<D>& st, const u32x4 (&p)[2], const char* values, int v0) {
#pragma unroll
  for (int u = 0; u < 2; ++u)                       // 16 keys an instruction
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {              // (8 and 16 rows further: the same swizzle)
      const char* at = values + (v0 ^ v_step(64 * d)) + u * 16 * 2 * D;
      const u32x2 lo = read_transposed(at), hi = read_transposed(at + 8 * 2 * D);
      st.acc[d] = Mfma<E>::m32(u32x4{lo[0], lo[1], hi[0], hi[1]}, p[u], st.acc[d]);
    }
}

// Values that are not finite, in the tiles t0 .. t1 - 1 that some row sees in part, tokens `from` .. to - 1 of each.
template <typename E, int D, bool kPaged, typename Sees>
__device__ __forceinline__ void add_odd(WideState<D>& st, const AttnArgs& a, const Seq& s, const Span& span, int b, int hk, int i0, int i1,
                                     int t0, int t1, int from, int to, int half, Sees sees) {
  using L = PageLayout<D>;
  const char* vb = a.v.data + 2 * (b * a.v.b + hk * a.v.h);
  for (int t = t0; t < t1; ++t) {
    bool cached;
    const int at = tile_of<kPage, 64>(span, t, &cached), n = min(64, (cached ? s.ctx : s.nk) - at);
    const uint8_t* page = kPaged && cached ? page_of(a.kv, b, at / kPage, hk) : nullptr;
    if (cached ? page == nullptr || full_cached(a, s, i1, at, 64) : full_new(a, s, i0, i1, at, 64)) continue;
    const uint64_t seen = sees(cached, at);
    for (int token = from; token < min(n, to); ++token) {
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4 v;
          if (kPaged && cached) {
            const float x = page[L::kVs + token * L::kScales + d] == 255 ? __builtin_nanf("") : 0.f;
            v = f32x4{x, x, x, x};
          } else {
            v = unclean<E>(vb + 2 * ((at + token) * a.v.t + 32 * d + 8 * e + 4 * half));
          }
          if ((seen >> token) & 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) st.acc[d][4 * e + k] += v[k];
        }
    }
  }
}

// The row's result, or its part of it.
template <typename E, int D>
__device__ __forceinline__ void wide_finish(const WideState<D>& st, const AttnArgs& a, const Split& sp, int b, int hk, int r, int i, int h,
                                            int half, int split) {
  const float l = st.l;
  if (sp.n == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char* dst = a.out.data + 2 * (b * a.out.b + i * a.out.t + h * a.out.h);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x16& x = st.acc[d];
        const u32x2 y = {E::pair(x[4 * e] * inv, x[4 * e + 1] * inv), E::pair(x[4 * e + 2] * inv, x[4 * e + 3] * inv)};
        *reinterpret_cast<u32x2*>(dst + 2 * (32 * d + 8 * e + 4 * half)) = y;
      }
    if (a.lse && half == 0)
      a.lse[((int64_t)b * a.T + i) * a.Hq + h] = l == 0.f ? -INFINITY : (st.m - E::kBias + __builtin_amdgcn_logf(l)) * kLn2;
  } else {
    const int64_t to = part_of(a, sp, b, hk, r) + split;
    if (half == 0) {
      sp.ml[2 * to] = st.m;
      sp.ml[2 * to + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(sp.sum + to * D + 32 * d + 8 * e + 4 * half) =
            f32x4{st.acc[d][4 * e], st.acc[d][4 * e + 1], st.acc[d][4 * e + 2], st.acc[d][4 * e + 3]};
  }
}

// 33 to 64 rows over a cache: two wavefront pairs share the rows out and take half of a tile's keys each, whose sums they join at
// the end.  Two tiles are on their way in registers (a tile's codes are a few) while one is in LDS.  A block of 16 with 4
// heads a kv head over 131072 cached tokens of 128 channels takes 64 us, 2.2 TB/s: a tile's chain of conversion, LDS,
// products and softmax between two barriers takes longer than its bytes, matrix units and vector units being busy 24% and
// 38% of the time and wavefronts waiting 42% of theirs.
template <typename E, int D>
__global__ __launch_bounds__(256, 2) void pair_kernel(AttnArgs a, Split sp) {
  constexpr int kTile = 64 * 2 * D;
  __shared__ __align__(16) char lds[2][2 * kTile];  // two tiles, keys then values: one is read while the next is written
  __shared__ uint32_t odd;                          // a tile not seen in full had values that are not finite
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.G;
  if (R == 0) return;
  const int i0 = 0, i1 = s.nq - 1;
  const Span span = span_of<kPage, 64>(a, s, i0, i1);
  const int per = ceil_div(span.n, sp.n), t0 = split * per, t1 = min(span.n, t0 + per);
  const int nc = max(t0, min(t1, span.a + span.c - span.b));   // this split's cached tiles come first

  const int r = 32 * (wave & 1) + col, rr = min(r, R - 1), i = rr / a.G, h = hk * a.G + rr % a.G;
  const int u0 = wave >> 1;                         // its 32-key part
  const bool mine = 32 * (wave & 1) < R;            // this wavefront has rows
  const RowAt row = row_at(a, s, b, i);
  u32x4 q[D / 16];
  {
    const u32x4* p = reinterpret_cast<const u32x4*>(a.q.data + 2 * (b * a.q.b + i * a.q.t + h * a.q.h + half * 8));
#pragma unroll
    for (int j = 0; j < D / 16; ++j) q[j] = signed_queries(p[2 * j], a.scale);
  }
  WideState<D> st;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) st.acc[t][e] = 0.f;
  const int k0 = k_at<D>(32 * u0 + col, half);
  const int v0 = v_at<D>(32 * u0 + 4 * half + (lane & 15) / 4, ((lane >> 4) & 1) * 32 + (lane & 3) * 8);
  const int shift = 4 * half + 32 * u0;             // a lane's first key in a tile
  const float c = score_factor(a.scale);
  if (tid == 0) odd = 0;
  __syncthreads();
  const char* kb = a.k.data + 2 * (b * a.k.b + hk * a.k.h);
  const char* vb = a.v.data + 2 * (b * a.v.b + hk * a.v.h);
  auto sees = [&](bool cached, int at) -> uint64_t {
    if (cached) return sees_cached(a, s, row).at(at);
    if (a.order == CADDTREE_ORDER_TREE) return sees_tree(a, s, b, row, at);
    return sees_new(a, s, row).at(at);
  };
  auto take = [&](const char* tile, bool full, uint32_t seen) {
    f32x16 x[1];
    wide_scores<E, D, 1>(x, q, tile, k0);
    u32x4 p[2];
    wide_raise<E, D, 1>(st, x, c, full, seen);
    wide_weights<E, D>(st, x[0], p, c);
    wide_values<E, D>(st, p, tile + kTile, v0);
  };

  int t = t0, buf = 0;
  bool cached;
  {
    struct Stage {
      PagePart<D> x;
      const uint8_t* page;
    } a0, a1;
    auto entry = [&](int tile) -> int32_t {
      return tile < nc ? table_entry(a.kv, b, tile_of<kPage, 64>(span, tile, &cached) / kPage) : -1;
    };
    auto load = [&](Stage& g, int32_t e) {
      g.page = page_at(a.kv, e, hk);
      g.x.load(g.page, tid);
    };
    auto full_at = [&](int here, bool there) { return there && full_cached(a, s, i1, here, 64); };
    auto store = [&](Stage& g, int tile, int to) {
      const int here = tile_of<kPage, 64>(span, tile, &cached);
      g.x.template store<E>(lds[to], lds[to] + kTile, tid, full_at(here, g.page), g.page ? s.ctx - here : 0, &odd);
    };
    int32_t ahead = -1;
    bool there = false;                             // the tile in LDS has a page
    if (t < nc) {
      const int32_t e0 = entry(t), e1 = entry(t + 1), e2 = entry(t + 2);
      ahead = entry(t + 3);
      load(a0, e0);
      load(a1, e1);
      store(a0, t, 0);
      there = a0.page;
      load(a0, e2);
      __syncthreads();
    }
    auto step = [&](Stage& g) {                     // tile t is in LDS, t + 1 in g
      if (mine) {
        const int here = tile_of<kPage, 64>(span, t, &cached);
        const bool full = full_at(here, there);
        take(lds[buf], full, full || !there ? 0 : (uint32_t)(sees(true, here) >> shift));
      }
      if (t + 1 < nc) {
        store(g, t + 1, buf ^ 1);
        there = g.page;
        load(g, ahead);
        ahead = entry(t + 4);
      }
      __syncthreads();
      buf ^= 1;
      ++t;
    };
    while (t < nc) {
      step(a1);
      if (t < nc) step(a0);
    }
  }
  {
    TensorPart<D> k, v;
    auto load = [&](int tile) {
      if (tile >= t1) return;
      const int here = tile_of<kPage, 64>(span, tile, &cached);
      k.load(kb, a.k.t, here, s.nk, tid);
      v.load(vb, a.v.t, here, s.nk, tid);
    };
    auto store = [&](int tile, int to) {
      const int here = tile_of<kPage, 64>(span, tile, &cached);
      k.store_keys(lds[to], tid);
      v.template store_values<E>(lds[to] + kTile, tid, full_new(a, s, i0, i1, here, 64), s.nk - here, &odd);
    };
    if (t < t1) {
      load(t);
      store(t, buf);
      load(t + 1);
      __syncthreads();
    }
    for (; t < t1; ++t) {
      if (mine) {
        const int here = tile_of<kPage, 64>(span, t, &cached);
        const bool full = full_new(a, s, i0, i1, here, 64);
        take(lds[buf], full, full ? 0 : (uint32_t)(sees(false, here) >> shift));
      }
      if (t + 1 < t1) {
        store(t + 1, buf ^ 1);
        load(t + 2);
      }
      __syncthreads();
      buf ^= 1;
    }
  }
  __syncthreads();
  if (odd && mine) add_odd<E, D, true>(st, a, s, span, b, hk, i0, i1, t0, t1, 32 * u0, 32 * u0 + 32, half, sees);
  st.l += __shfl_xor(st.l, 32);
  {                                                 // the second pair's sums to the first, 16 registers at a time
    __syncthreads();
    float* box = reinterpret_cast<float*>(lds) + (wave & 1) * 1024 + lane;   // 2 x 64 lanes x 16 values, the lanes side by side
    float* box_ml = reinterpret_cast<float*>(lds) + 2 * 1024 + (wave & 1) * 128 + lane;
    if (wave >= 2) {
      box_ml[0] = st.m;
      box_ml[64] = st.l;
    }
    __syncthreads();
    const float m2 = box_ml[0], l2 = box_ml[64], m = fmaxf(st.m, m2);
    const float f1 = st.l == 0.f ? 0.f : st.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
    const float f2 = l2 == 0.f ? 0.f : m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2 - m);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      if (wave >= 2)
#pragma unroll
        for (int e = 0; e < 16; ++e) box[64 * e] = st.acc[d][e];
      __syncthreads();
      if (wave < 2)
#pragma unroll
        for (int e = 0; e < 16; ++e) st.acc[d][e] = st.acc[d][e] * f1 + box[64 * e] * f2;
      __syncthreads();
    }
    if (wave >= 2) return;
    st.l = st.l * f1 + l2 * f2;
    st.m = m;
  }
  if (r < R) wide_finish<E, D>(st, a, sp, b, hk, r, i, h, half, split);
}

// 128 rows a workgroup, 32 a wavefront.  Bound by the matrix products and by forming the weights, which hardly overlap:
// at 128 channels a tile takes a wavefront 32 products (1024 cycles) and some 230 vector instructions, 32 of them
// exponentials (1300 cycles), of the 2500 it takes in all.  A prompt of 8192 tokens of 32 heads through a window of 2048
// takes 276 us (873 TFLOP/s; matrix units busy 46%, vector units 48% of the time); 32 trees of 257 rows over 4096 cached
// tokens take 618 us (713 TFLOP/s): there a tile is converted on its way into LDS and the wavefronts wait 45% of their
// time, 23% where tiles go straight to LDS.  The next tile stored earlier (before this one or between its scores and its
// softmax), or loaded a tile earlier, took 1 to 3% longer; eight wavefronts or 64 rows a wavefront that share a tile,
// tiles of 32 keys with three wavefronts a SIMD, priorities for the products, or half tiles interleaved, the same or more.
template <typename E, int D, bool kPaged>
__global__ __launch_bounds__(256, 2) void wide_kernel(AttnArgs a, Split sp) {
  constexpr int kRows = 128, kTile = 64 * 2 * D, kHalf = 32 * 2 * D;
  __shared__ __align__(16) char lds[2][2 * kTile];  // two tiles, keys then values: one is read while the next is written
  __shared__ uint32_t odd;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
  // Workgroups go to the eight dies in turn, and each die has its own L2: a sequence and kv head's workgroups, which
  // read the same keys, are those of one die (a windowed prompt of 8192: 405 -> 372 us).
  const int parts = ((a.T * a.G + kRows - 1) / kRows) * sp.n, pair = blockIdx.x / (8 * parts) * 8 + blockIdx.x % 8;
  if (pair >= a.B * a.Hkv) return;
  const int part = blockIdx.x / 8 % parts, split = part % sp.n, tile_row = part / sp.n, hk = pair % a.Hkv, b = pair / a.Hkv;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.G, r0 = tile_row * kRows;
  if (r0 >= R) return;
  const int i0 = r0 / a.G, i1 = min(R - 1, r0 + kRows - 1) / a.G;
  const Span span = span_of<kPage, 64>(a, s, i0, i1);
  const int per = ceil_div(span.n, sp.n), t0 = split * per, t1 = min(span.n, t0 + per);
  const int nc = kPaged ? max(t0, min(t1, span.a + span.c - span.b)) : t0;   // this split's cached tiles come first

  const int r = r0 + 32 * wave + col, rr = min(r, R - 1), i = rr / a.G, h = hk * a.G + rr % a.G;
  const bool mine = r0 + 32 * wave < R;             // this wavefront has rows
  const RowAt row = row_at(a, s, b, i);
  u32x4 q[D / 16];
  {
    const u32x4* p = reinterpret_cast<const u32x4*>(a.q.data + 2 * (b * a.q.b + i * a.q.t + h * a.q.h + half * 8));
#pragma unroll
    for (int j = 0; j < D / 16; ++j) q[j] = signed_queries(p[2 * j], a.scale);
  }
  WideState<D> st;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) st.acc[t][e] = 0.f;
  const int k0 = k_at<D>(col, half);
  const int v0 = v_at<D>(4 * half + (lane & 15) / 4, ((lane >> 4) & 1) * 32 + (lane & 3) * 8);
  const float c = score_factor(a.scale);
  if (tid == 0) odd = 0;
  __syncthreads();
  const char* kb = a.k.data + 2 * (b * a.k.b + hk * a.k.h);
  const char* vb = a.v.data + 2 * (b * a.v.b + hk * a.v.h);
  auto sees = [&](bool cached, int at) -> uint64_t {
    if (kPaged && cached) return sees_cached(a, s, row).at(at);
    if (kPaged && a.order == CADDTREE_ORDER_TREE) return sees_tree(a, s, b, row, at);
    return sees_new(a, s, row).at(at);
  };
  auto take = [&](const char* tile, bool full, uint64_t seen) {
    f32x16 x[2];
    wide_scores<E, D, 2>(x, q, tile, k0);
    wide_raise<E, D, 2>(st, x, c, full, seen);
    u32x4 p0[2], p1[2];
    wide_weights<E, D>(st, x[0], p0, c);
    wide_values<E, D>(st, p0, tile + kTile, v0);
    wide_weights<E, D>(st, x[1], p1, c);
    wide_values<E, D>(st, p1, tile + kTile + kHalf, v0);
  };

  int t = t0, buf = 0;
  bool cached;
  if constexpr (kPaged) {
    PagePart<D> x;
    const uint8_t* page = nullptr;
    auto entry = [&](int tile) -> int32_t {
      return tile < nc ? table_entry(a.kv, b, tile_of<kPage, 64>(span, tile, &cached) / kPage) : -1;
    };
    auto load = [&](int32_t e) {
      page = page_at(a.kv, e, hk);
      x.load(page, tid);
    };
    auto full_at = [&](int here, bool there) { return there && full_cached(a, s, i1, here, 64); };
    auto store = [&](int tile, int to) {
      const int here = tile_of<kPage, 64>(span, tile, &cached);
      x.template store<E>(lds[to], lds[to] + kTile, tid, full_at(here, page), page ? s.ctx - here : 0, &odd);
    };
    int32_t ahead = -1;
    bool there = false;                             // the tile in LDS has a page
    if (t < nc) {
      const int32_t e0 = entry(t), e1 = entry(t + 1);
      ahead = entry(t + 2);
      load(e0);
      store(t, 0);
      there = page;
      load(e1);
      __syncthreads();
    }
    for (; t < nc; ++t) {
      if (mine) {
        const int here = tile_of<kPage, 64>(span, t, &cached);
        const bool full = full_at(here, there);
        take(lds[buf], full, full || !there ? 0 : sees(true, here) >> (4 * half));
      }
      if (t + 1 < nc) {
        store(t + 1, buf ^ 1);
        there = page;
        load(ahead);
        ahead = entry(t + 3);
      }
      __syncthreads();
      buf ^= 1;
    }
  }
  {
    // A tile seen in full goes straight to LDS while the one before it is taken; the others pass through registers,
    // where values that are not to count are taken out.
    TensorPart<D> k, v;
    const TileMove<D> km(a.k.t, tid, wave, true), vm(a.v.t, tid, wave, false);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0];
    bool whole = false;
    auto begin = [&](int tile, int to) {
      const int here = tile_of<kPage, 64>(span, tile, &cached);
      whole = full_new(a, s, i0, i1, here, 64);
      if (whole) {
        km.send(kb, a.k.t, here, lds0 + to * 2 * kTile);
        vm.send(vb, a.v.t, here, lds0 + to * 2 * kTile + kTile);
      } else {
        k.load(kb, a.k.t, here, s.nk, tid);
        v.load(vb, a.v.t, here, s.nk, tid);
      }
    };
    auto end = [&](int tile, int to) {
      if (!whole) {
        const int here = tile_of<kPage, 64>(span, tile, &cached);
        k.store_keys(lds[to], tid);
        v.template store_values<E>(lds[to] + kTile, tid, false, s.nk - here, &odd);
      }
      tiles_there();
    };
    if (t < t1) {
      begin(t, buf);
      end(t, buf);
      __syncthreads();
    }
    for (; t < t1; ++t) {
      const bool full = whole;
      if (t + 1 < t1) begin(t + 1, buf ^ 1);
      if (mine) take(lds[buf], full, full ? 0 : sees(false, tile_of<kPage, 64>(span, t, &cached)) >> (4 * half));
      if (t + 1 < t1) end(t + 1, buf ^ 1);
      __syncthreads();
      buf ^= 1;
    }
  }
  __syncthreads();
  if (odd && mine) add_odd<E, D, kPaged>(st, a, s, span, b, hk, i0, i1, t0, t1, 0, 64, half, sees);
  st.l += __shfl_xor(st.l, 32);
  if (r < R) wide_finish<E, D>(st, a, sp, b, hk, r, i, h, half, split);
}

// Joins the splits of a row, few of them: D / 4 lanes a row, 4 channels each.  Two loads deep and bound by their latency:
// 3 us for 256 rows of 5 splits.
template <typename E>
__device__ void write_row(const AttnArgs& a, int b, int hk, int r, int ch, f32x4 o, float m, float l) {
  const int i = r / a.G, h = hk * a.G + r % a.G;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(a.out.data + 2 * (b * a.out.b + i * a.out.t + h * a.out.h + 4 * ch)) =
      u32x2{E::pair(o[0] * inv, o[1] * inv), E::pair(o[2] * inv, o[3] * inv)};
  if (a.lse && ch == 0)
    a.lse[((int64_t)b * a.T + i) * a.Hq + h] = l == 0.f ? -INFINITY : (m - E::kBias + __builtin_amdgcn_logf(l)) * kLn2;
}
// a split's factor for the row's maximum m (a split without a key left its sums unset)
__device__ inline float split_factor(float mk, float lk, float m) {
  return lk == 0.f ? 0.f : mk == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mk - m);
}
template <typename E, int D>
__global__ __launch_bounds__(256) void combine_few_kernel(AttnArgs a, Split sp) {
  constexpr int kLanes = D / 4;
  const int ch = threadIdx.x % kLanes, hk = blockIdx.y, b = blockIdx.z;
  const int64_t r = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const Seq s = sequence(a, b);
  if (r >= (int64_t)s.nq * a.G) return;
  const int64_t at = part_of(a, sp, b, hk, (int)r);
  float mk[kFewSplits], lk[kFewSplits], m = -INFINITY, l = 0.f;
  f32x4 x[kFewSplits], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {            // (all loads in flight; a split that is not there reads the first)
    const int64_t p = at + (k < sp.n ? k : 0);
    mk[k] = sp.ml[2 * p];
    lk[k] = k < sp.n ? sp.ml[2 * p + 1] : 0.f;
    x[k] = *reinterpret_cast<const f32x4*>(sp.sum + p * D + 4 * ch);
    m = fmaxf(m, mk[k]);
  }
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {
    const float f = split_factor(mk[k], lk[k], m);
    l += lk[k] * f;
    if (lk[k] != 0.f) o += f * x[k];
  }
  write_row<E>(a, b, hk, (int)r, ch, o, m, l);
}
// ... many of them: a workgroup a row.  Its threads look at a split each for the maximum, the sum and the factors;
// then groups of D / 4 lanes take every n-th split's sums and add up through LDS, in a fixed order.  512 rows of 64
// splits: 6 us (17 MB, 2.8 TB/s); with a group of lanes a row as above the whole call took 87 us in place of 74.
template <typename E, int D>
__global__ __launch_bounds__(256) void combine_many_kernel(AttnArgs a, Split sp) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float factor[kMaxSplits], top[4], total[4];
  __shared__ __align__(16) f32x4 part[256];
  const int tid = threadIdx.x, r = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const Seq s = sequence(a, b);
  if (r >= (int64_t)s.nq * a.G) return;
  const int64_t at = part_of(a, sp, b, hk, r);
  float mk[2], lk[2], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int k = tid + 256 * j;
    mk[j] = k < sp.n ? sp.ml[2 * (at + k)] : -INFINITY;
    lk[j] = k < sp.n ? sp.ml[2 * (at + k) + 1] : 0.f;
    m = fmaxf(m, mk[j]);
  }
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (tid % 64 == 0) top[tid / 64] = m;
  __syncthreads();
  m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float f = split_factor(mk[j], lk[j], m);
    if (tid + 256 * j < sp.n) factor[tid + 256 * j] = lk[j] == 0.f ? -1.f : f;      // (-1: its sums are unset)
    l += lk[j] * f;
  }
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  if (tid % 64 == 0) total[tid / 64] = l;
  __syncthreads();
  l = (total[0] + total[1]) + (total[2] + total[3]);
  const int ch = tid % kLanes, group = tid / kLanes;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = group; k < sp.n; k += kGroups) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(sp.sum + (at + k) * D + 4 * ch);
    const float f = factor[k];
    if (f != -1.f) o += f * x;
  }
  part[tid] = o;
  __syncthreads();
  if (group != 0) return;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) o += part[tid + g * kLanes];
  write_row<E>(a, b, hk, r, ch, o, m, l);
}

template <typename E, int D, bool kPaged>
hipError_t launch(const AttnArgs& a, const Split& sp, hipStream_t stream) {
  const int64_t R = (int64_t)a.T * a.G;
  const dim3 few(sp.n, a.Hkv, a.B);
  bool done = false;
  if constexpr (kPaged) {
    done = R <= 64;
    if (R <= 16) narrow_kernel<E, D, 1, true><<<few, 256, 0, stream>>>(a, sp);
    else if (R <= 32) narrow_kernel<E, D, 2, true><<<few, 256, 0, stream>>>(a, sp);
    else if (R <= 64) pair_kernel<E, D><<<few, 256, 0, stream>>>(a, sp);
  } else if (R <= 16) {
    const int64_t reach = a.window == 0 ? a.S : std::min<int64_t>(a.S, (int64_t)a.window + a.sinks + a.T);
    done = reach * a.Hkv * a.B <= kFewKeys;
    if (done) narrow_kernel<E, D, 1, false><<<few, 256, 0, stream>>>(a, sp);
  }
  if (!done)
    wide_kernel<E, D, kPaged><<<dim3((unsigned)((R + 127) / 128 * sp.n * (((int64_t)a.B * a.Hkv + 7) / 8 * 8))), 256, 0, stream>>>(a, sp);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.n == 1) return e;
  const int lanes = D / 4;
  if (sp.n <= kFewSplits) combine_few_kernel<E, D><<<dim3((unsigned)((R * lanes + 255) / 256), a.Hkv, a.B), 256, 0, stream>>>(a, sp);
  else combine_many_kernel<E, D><<<dim3((unsigned)R, a.Hkv, a.B), 256, 0, stream>>>(a, sp);
  return hipGetLastError();
}

template <typename E, int D>
hipError_t launch(const AttnArgs& a, const Split& sp, hipStream_t stream) {
  return a.kv.pages ? launch<E, D, true>(a, sp, stream) : launch<E, D, false>(a, sp, stream);
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, const Split& sp, caddtree_dtype_t dtype, int32_t D, hipStream_t stream) {
  if (dtype == CADDTREE_BF16) return D == 64 ? launch<BF16, 64>(a, sp, stream) : launch<BF16, 128>(a, sp, stream);
  return D == 64 ? launch<F16, 64>(a, sp, stream) : launch<F16, 128>(a, sp, stream);
}

}  // namespace caddtree
