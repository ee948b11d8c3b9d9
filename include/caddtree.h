/*
 * caddtree.h -- C ABI of the CaDDTree draft-tree construction library (MI355X / gfx950).
 *
 * What it computes (Cost-Aware Diffusion Draft Trees for Speculative Decoding,
 * arXiv 2606.01813):  a speculative-decoding round starts from a block-diffusion
 * drafter's logits l_1 .. l_L over a vocabulary of V tokens.  Per round the
 * library
 *   1. forms the full-vocabulary log-normaliser LSE_i and the top-K tokens of
 *      every position i with log q_i^(k) = l_i^(k) - LSE_i (Sec. 3.2, eq.
 *      marginals; the Require line of Algorithm 1);
 *   2. grows the draft tree best-first by prefix probability pi_s =
 *      prod_i q_i(s_i) (eq. prefix-prob) and stops at the first budget n where
 *      theta*(n) = (1 + Phi*(n)) / (C_d + C_v(n)) (eq. per-round) stops rising
 *      (Algorithm 1; Lemma 1, eq. stopping; Cor. 2);
 *   3. lays the tree out breadth-first and emits its tree-attention mask
 *      (each node sees itself and its ancestors, Sec. 3.3) and position ids.
 *
 * Conventions shared by every entry point:
 *   - Device pointers are HIP device memory on the plan's device; host pointers
 *     are named *_host.  The caller owns every buffer; the library allocates
 *     nothing per call (a plan owns one small device copy of its cost tables
 *     and context-length grid).
 *   - All work is enqueued on the given stream and runs asynchronously; the
 *     return value reports argument validation (done synchronously, before
 *     anything is enqueued) and launch errors, not kernel completion.
 *   - A non-OK status enqueues nothing new; caddtree_last_error() gives a
 *     message (thread-local).  No C++ exception crosses this interface.
 *   - Logits must be finite; results for NaN or +-Inf inputs are unspecified.
 *   - Layouts are row-major.  B rounds, L positions, V vocabulary, K kept tokens
 *     per position, cap = budget cap.  Logit row (b, i) starts at element
 *     (b * L + i) * row_stride, row_stride >= V elements.
 *   - Output slots at or beyond a round's n_star are left untouched; consumers
 *     read n_star.  n_star = 0 (an empty tree) is a legal result.
 *
 * Tie-breaking (the paper leaves it open; fixed here so results are unique):
 *   - top-K: value descending, then token id ascending;
 *   - expansion order: log prefix probability descending, then depth
 *     ascending, then the sum of raw logits along the path descending, then
 *     the rank tuple lexicographically ascending;
 *   - stop: theta_new <= theta_prev stops (ties keep the smaller tree), as in
 *     Algorithm 1;
 *   - output order: depth ascending, then rank tuple lexicographically
 *     ascending (parents precede children).
 */
#ifndef CADDTREE_H
#define CADDTREE_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CADDTREE_MAX_L 32
#define CADDTREE_MAX_K 16
#define CADDTREE_MAX_CAP 4096
#define CADDTREE_MAX_CTX 64     /* context-length grid points */

typedef enum {
  CADDTREE_OK = 0,
  CADDTREE_E_INVALID = 1,      /* bad argument: NULL where required, negative or inconsistent size */
  CADDTREE_E_UNSUPPORTED = 2,  /* valid request beyond the library's limits (L, K, cap, V) */
  CADDTREE_E_COST = 3,         /* cost model rejected: C_d <= 0, non-finite, C_v decreasing or not convex */
  CADDTREE_E_WORKSPACE = 4,    /* workspace NULL, misaligned or too small for the top-K table */
  CADDTREE_E_HIP = 5           /* a HIP runtime call or kernel launch failed */
} caddtree_status_t;

/* Logits are F32 or BF16; the attention operators below take BF16 or F16, the operators on logits all three. */
typedef enum { CADDTREE_F32 = 0, CADDTREE_BF16 = 1, CADDTREE_F16 = 2 } caddtree_dtype_t;

/* Tree-attention mask format.  U8: [B, cap, cap] bytes, mask[b][i][j] = 1 iff
 * node j is node i or an ancestor of i.  BITS32: [B, cap, ceil(cap/32)] u32
 * words, bit (j % 32) of word (j / 32), least significant bit first.  Only
 * rows i < n_star and columns j < n_star (words j/32 < ceil(n_star/32)) are
 * written; for BITS32 the bits of the last written word at or beyond n_star
 * are written as zero. */
typedef enum { CADDTREE_MASK_NONE = 0, CADDTREE_MASK_U8 = 1, CADDTREE_MASK_BITS32 = 2 } caddtree_mask_t;

/* flags */
#define CADDTREE_ALLOW_NONCONVEX 1u  /* accept a C_v that is non-decreasing but not convex (Assumption 1
                                        may then fail: the greedy stop is still taken, optimality is not claimed) */
#define CADDTREE_FIXED_BUDGET 2u     /* fixed-budget mode (the DDTree construction, Sec. 3.4): no stop rule;
                                        every round keeps the top min(budget_cap, sum_d K^d) nodes by prefix
                                        probability, in the same order and layout.  phi and theta are still
                                        reported, theta from the plan's cost model at that size. */

typedef struct caddtree_plan* caddtree_plan_t;   /* opaque, immutable after creation */

/* Static description of a workload. */
typedef struct {
  int32_t L;                 /* block positions, 1 .. CADDTREE_MAX_L */
  int64_t V;                 /* vocabulary size, K .. 2^31 - 1 */
  int32_t K;                 /* tokens kept per position, 1 .. CADDTREE_MAX_K */
  int32_t budget_cap;        /* maximum nodes per tree, 0 .. CADDTREE_MAX_CAP */
  caddtree_dtype_t dtype;    /* logits element type */
  caddtree_mask_t mask;      /* mask format written by caddtree_build / caddtree_emit */
  uint32_t flags;            /* CADDTREE_ALLOW_NONCONVEX | CADDTREE_FIXED_BUDGET, or 0 */
  double t_draft;            /* C_d > 0, drafting cost of one round (Sec. 4.2) */
  const double* t_verify_host; /* HOST array of max(n_ctx, 1) x (budget_cap + 1) values: row j is
                                  C_v(0 .. cap; L_j), the verification cost of a tree of n nodes at
                                  context length L_j (Sec. 4.2, Sec. 4.6).  Every row must be finite,
                                  non-decreasing and convex in n (Cor. 3) up to a relative rounding
                                  slack of 1e-12; copied at plan creation. */
  int32_t n_ctx;             /* J, context-length grid points: 0 or 1 = one cost table and no context
                                dependence (ctx_len is then ignored); 2 .. CADDTREE_MAX_CTX = one table
                                per grid point, interpolated per round (Sec. 4.6, eq. cv-interp) */
  const int64_t* ctx_grid_host; /* HOST, J context lengths 0 <= L_0 < L_1 < ... < L_{J-1} <= 2^53
                                   (used when J >= 2); copied at plan creation */
} caddtree_config_t;

/* Validates cfg, copies the cost table to the current device and returns a plan.
 * The plan holds what Algorithm 1 takes besides the marginals: K, the costs C_d
 * and C_v(n; l) of Sec. 4.2 / 4.6 (eq. per-round's denominator), with the budget
 * cap this library adds, and the launch layout.  Rejects a cost that breaks
 * Assumption 1 (C_v non-decreasing and convex, Cor. 3) with CADDTREE_E_COST.
 * The plan is bound to the device that is current at creation; *plan_out is
 * NULL on any error.  Not thread-safe against caddtree_plan_destroy of the
 * same plan; concurrent builds on one plan are safe (distinct outputs and
 * workspaces). */
caddtree_status_t caddtree_plan_create(const caddtree_config_t* cfg, caddtree_plan_t* plan_out);
/* Frees the plan (NULL is a no-op).  The caller ensures no enqueued work still uses it. */
void caddtree_plan_destroy(caddtree_plan_t plan);

/* Device workspace caddtree_build uses for up to B rounds: the top-K table when
 * the caller does not ask for it, and for a few rounds the partial results of
 * rows that several workgroups reduce (a workspace that holds the table alone is
 * accepted; such a call reduces a row in one workgroup, and the last bits of its
 * normalisers may differ).  It never falls as B grows.  256-byte alignment is
 * required. */
size_t caddtree_workspace_bytes(caddtree_plan_t plan, int64_t B);

/* Outputs of caddtree_build (DEVICE pointers).  Required: token_ids, parent,
 * depth, n_star.  Optional (NULL skips the output): everything else.
 *   token_ids [B, cap] int32  vocabulary id of node i (canonical order)
 *   parent    [B, cap] int32  index of the parent node, -1 when the parent is the root (bonus token)
 *   depth     [B, cap] int32  1 .. L
 *   path_prob [B, cap] float  pi_s of the node (eq. prefix-prob), rounded to fp32
 *   n_star    [B]      int32  chosen budget
 *   phi       [B]      float  Phi*(n_star) = sum of path_prob over the tree (eq. surrogate), fp32
 *   theta     [B]      float  theta*(n_star) (eq. per-round), fp32
 *   mask      see caddtree_mask_t; ignored when the plan's mask is NONE
 *   pos_ids   [B, cap] int32  pos_offset + depth
 *   topk_ids  [B, L, K] int32, topk_logit [B, L, K] float (raw logits),
 *   topk_lq   [B, L, K] float (log q_i^(k)), lse [B, L] double (LSE_i) */
typedef struct {
  int32_t* token_ids;
  int32_t* parent;
  int32_t* depth;
  float* path_prob;
  int32_t* n_star;
  float* phi;
  float* theta;
  void* mask;
  int32_t* pos_ids;
  int32_t* topk_ids;
  float* topk_logit;
  float* topk_lq;
  double* lse;
} caddtree_outputs_t;

/* Context length of each round (plans with J >= 2 cost tables).  ctx_len is a
 * DEVICE int64 array [B].  A round at context length l with L_j <= l < L_{j+1}
 * uses C_v(n; l) = (1 - a) C_v(n; L_j) + a C_v(n; L_{j+1}), a = (l - L_j) /
 * (L_{j+1} - L_j) (eq. cv-interp), each product and the sum rounded
 * separately in fp64; l <= L_0 uses the L_0 table and l >= L_{J-1} the
 * L_{J-1} table (no extrapolation, which could break convexity).  NULL is an
 * error for such plans and is allowed otherwise. */

/* The whole hot path for B rounds (Sec. 3.2-3.3 and Algorithm 1): per round the
 * full-vocabulary log-normaliser and top-K of every position (eq. marginals),
 * the best-first expansion with the greedy stop of Lemma 1 (eq. stopping; the
 * tree T*_{n*} of eq. phistar at n* = the first maximiser of eq. per-round,
 * Cor. 2), and the tree-attention mask and position ids (Sec. 3.3).
 * logits: DEVICE [B, L, row_stride] of the plan's dtype; B >= 0 (0 is a no-op).
 * workspace: DEVICE, caddtree_workspace_bytes(plan, B) bytes, 256-byte aligned
 * (may be NULL when every top-K output pointer is given; one that is given is
 * then still used for the partial results of a few rounds).
 * The call only enqueues kernels on `stream` (no allocation, memset or
 * synchronisation), so it may be captured in a HIP graph; a replay reads and
 * writes the buffers given at capture. */
caddtree_status_t caddtree_build(caddtree_plan_t plan, const void* logits, int64_t B, int64_t row_stride,
                                 int32_t pos_offset, const int64_t* ctx_len, const caddtree_outputs_t* out,
                                 void* workspace, size_t workspace_bytes, hipStream_t stream);

/* For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): caddtree_build with no
 * workspace argument.  The top-K table the caller does not ask for lives in a
 * device array inside the library, CADDTREE_NOALLOC_SCRATCH_BYTES per GPU, held
 * until the process ends; the call allocates and frees nothing and runs the same
 * kernels as caddtree_build with a workspace, with the same results (as without
 * one when every top-K output is given: the array is then not used).
 *   Limit: the table of the top-K outputs left NULL must not exceed
 *   CADDTREE_NOALLOC_SCRATCH_BYTES (8 MiB: about
 *   2^20 / (L K + L) rounds, 7281 at L = 16, K = 8), else CADDTREE_E_WORKSPACE
 *   and nothing is enqueued.  Passing every top-K output lifts the limit.
 *   Every call on one GPU shares that GPU's array, whatever the plan or stream:
 *   calls that overlap in time on one GPU race (serialise them, e.g. on one
 *   stream).  Each call writes the part it reads before reading it, so nothing
 *   needs clearing between calls.
 *   Other arguments and errors as for caddtree_build; E_HIP if the array's
 *   address could not be taken when the plan was created. */
#define CADDTREE_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)
caddtree_status_t caddtree_build_noalloc(caddtree_plan_t plan, const void* logits, int64_t B, int64_t row_stride,
                                         int32_t pos_offset, const int64_t* ctx_len, const caddtree_outputs_t* out,
                                         hipStream_t stream);

/* Stage 1 (Sec. 3.2): per (round, position) row, LSE in fp64 and the top-K by
 * (value desc, id asc).  topk_ids, topk_logit, lse required; topk_lq optional.
 * A row is one workgroup's here at any batch, so the last bits of lse may differ
 * from those of a caddtree_build of a few rounds. */
caddtree_status_t caddtree_reduce_topk(caddtree_plan_t plan, const void* logits, int64_t B, int64_t row_stride,
                                       int32_t* topk_ids, float* topk_logit, float* topk_lq, double* lse,
                                       hipStream_t stream);

/* Stage 2 (Algorithm 1): best-first expansion with the greedy stop, tree in canonical order.
 * Inputs: topk_ids, topk_logit [B, L, K], lse [B, L] (DEVICE); ctx_len as for
 * caddtree_build.  token_ids, parent, depth, n_star required; path_prob, phi,
 * theta optional. */
caddtree_status_t caddtree_expand(caddtree_plan_t plan, const int32_t* topk_ids, const float* topk_logit,
                                  const double* lse, int64_t B, const int64_t* ctx_len,
                                  int32_t* token_ids, int32_t* parent, int32_t* depth, float* path_prob,
                                  int32_t* n_star, float* phi, float* theta, hipStream_t stream);

/* Stage 3 (Sec. 3.3): tree-attention mask and position ids from parent/depth/n_star.
 * mask may be NULL (or the plan's mask NONE) to skip it; pos_ids may be NULL. */
caddtree_status_t caddtree_emit(caddtree_plan_t plan, const int32_t* parent, const int32_t* depth,
                                const int32_t* n_star, int64_t B, int32_t pos_offset,
                                void* mask, int32_t* pos_ids, hipStream_t stream);

/* Synthetic acceptance (tree verification, Sec. 3.3) of B built trees against
 * target continuations drawn from the drafter's factorised distribution
 * (eq. factorized), under which the expected accepted length of a tree is
 * Phi (eq. surrogate).  For a simulated throughput sum (1 + alpha) / sum C
 * (Sec. 4.2) over many rounds.
 *   topk_ids, topk_logit [B, L, K], lse [B, L]: DEVICE, as written by stage 1
 *   token_ids, parent [B, tree_stride], n_star [B]: DEVICE, a tree as written
 *       by caddtree_build / caddtree_expand (tree_stride = the budget cap of
 *       the plan that built it; n_star is clamped to [0, tree_stride])
 *   u [B, L]: DEVICE fp64 uniforms in [0, 1), owned by the caller (the random
 *       numbers are inputs).  Position i draws rank r for the smallest r with
 *       u_i < q^(0) + .. + q^(r), q^(k) = exp(l^(k) - LSE_i), the sum formed
 *       left to right in fp64; u_i at or above the sum of all K draws a token
 *       outside the top-K, which no node carries.
 *   accept_len [B] int32 (required): the length of the longest drawn prefix
 *       that is a path of the tree, 0 .. L.
 *   round_cost [B] fp64 (optional): C_d + C_v(n_star; l) from THIS plan's cost
 *       model (which may differ from the one that built the trees), NaN when
 *       n_star lies outside [0, cap]; ctx_len as for caddtree_build. */
caddtree_status_t caddtree_accept(caddtree_plan_t plan, const int32_t* topk_ids, const float* topk_logit,
                                  const double* lse, int64_t B, const int32_t* token_ids, const int32_t* parent,
                                  int32_t tree_stride, const int32_t* n_star, const double* u,
                                  const int64_t* ctx_len, int32_t* accept_len, double* round_cost,
                                  hipStream_t stream);

/* HOST only (no GPU, no stream): the offline cost model of Sec. 4.6.  Fits a
 * verification-cost profile y_j measured at node counts x_j (x strictly
 * increasing, all finite, 1 <= N <= 2^22) by the least-squares function that
 * is convex and non-decreasing (eq. convex-reg): a piecewise-linear function
 * whose breakpoints the data choose, solved exactly (active-set non-negative
 * least squares on the slope changes).
 *   fit_host [N] (optional): the fitted values at the x_j;
 *   table_host [cap + 1] (optional, 0 <= cap <= CADDTREE_MAX_CAP): the fit at
 *       n = 0 .. cap, interpolated linearly between the x_j and continued
 *       along the end segments outside them, ready to be a plan's
 *       t_verify_host row (one fit per context length, Sec. 4.6).
 * Host memory for the solve is allocated internally.  Returns E_INVALID for
 * bad input and E_UNSUPPORTED if the iteration does not settle. */
caddtree_status_t caddtree_fit_cost(const double* x_host, const double* y_host, int64_t N, double* fit_host,
                                    int32_t cap, double* table_host);

/* ------------------------------------------------------------------------------------------------
 * Verification: the target's attention over a built tree, and the 4-bit cache it reads.
 *
 * After a build the target verifies the tree (Sec. 3.1, 3.3): the bonus token (the root) and the n_star
 * nodes are its queries, and each sees the cached context, the root, its ancestors and itself.  These
 * calls are that attention, the cache of keys and values in 4 bits behind it, the attention of a
 * prompt or of single tokens through a sliding window, and a cache's eviction by accumulated attention
 * weight.  They take no plan; they run on the current device, with the conventions at the top of this
 * file (asynchronous on `stream`, no allocation, arguments checked before anything is enqueued, fit for
 * HIP graph capture).  Lengths and page tables are DEVICE arrays and so are not checked: the kernels
 * clamp a length to what its buffer holds, and a page number outside the cache holds no key.
 *
 * Tensors of 16-bit elements are strided views [B, tokens, heads, head_dim]: element (b, t, h, d) at
 * data + b stride_b + t stride_t + h stride_h + d (strides in elements).  data must be 16-byte aligned
 * and the strides multiples of 8, stride_t below 2^24; inputs may overlap or repeat (stride 0).
 *
 * Visibility.  Query i at position pos_i sees the key at position pos_j if its order allows it and
 *     window = 0  or  pos_i - pos_j < window  or  pos_j < sinks.
 * Positions in a cache are slot numbers.  After an eviction (caddtree_cache_evict) the kept slots lie next to
 * each other, so a window counts kept slots, not the tokens that were between them.
 * An absent key never sees use: whatever its memory holds (NaN included) does not reach a result, and
 * what a query does not see does not reach its row.  A query that sees no key gets zeros and
 * lse = -inf.
 *     s_ij = scale q_i . k_j       lse_i = log sum_visible exp(s_ij)       out_i = sum_visible exp(s_ij - lse_i) v_j
 * Products are formed on 16-bit inputs and summed in fp32; the softmax is fp32; a weight is rounded to
 * the inputs' type for its product with v. */
typedef struct {
  void* data;
  int64_t stride_b, stride_t, stride_h;
} caddtree_view_t;

/* How the new keys (those given as tensors) are ordered for the queries. */
typedef enum {
  CADDTREE_ORDER_CHAIN = 0,  /* causal: pos_j <= pos_i */
  CADDTREE_ORDER_BLOCK = 1,  /* every query sees every key (a block-diffusion drafter's block) */
  CADDTREE_ORDER_TREE = 2    /* a draft tree's mask: query 0 is the root, query i node i - 1 */
} caddtree_order_t;

#define CADDTREE_PAGE 64     /* tokens of a cache page */
#define CADDTREE_KV_BLOCK 32 /* channels that share a scale */

/* A cache of keys and values in 4 bits: n_pages pages of CADDTREE_PAGE tokens, laid out
 * [n_pages, n_kv_heads, CADDTREE_PAGE_BYTES(head_dim)].  The bytes of a page and head:
 *     key codes [64, head_dim / 2], value codes [64, head_dim / 2],
 *     key scales [64, head_dim / 32], value scales [64, head_dim / 32].
 * A value is code x 2^(scale - 127): the code is a sign bit and one of 0 0.5 1 1.5 2 3 4 6 (E2M1), an
 * even channel in the low half of its byte; the scale byte is a power of two for 32 channels, 255 for
 * a block that holds a NaN or an infinity (all 32 of its values are then NaN).  Slot t of sequence b
 * lives in page page_table[b, t / 64] at token t % 64.  `dtype` is the type of the keys and values
 * written and of the queries: scales are kept where every value is a normal number of that type
 * (exponents -125 .. 125 in BF16, -13 .. 13 in F16; larger values saturate, smaller ones round on that
 * grid). */
#define CADDTREE_PAGE_BYTES(head_dim) ((int64_t)68 * (head_dim))
typedef struct {
  caddtree_dtype_t dtype;   /* BF16 or F16 */
  int32_t n_kv_heads;
  int32_t head_dim;         /* 64 or 128 */
  int64_t n_pages;
  void* pages;              /* DEVICE, 256-byte aligned */
} caddtree_cache_t;

/* One attention call: queries, new keys and values, and for the cached form the sequences' pages. */
typedef struct {
  caddtree_dtype_t dtype;       /* BF16 or F16 */
  int32_t B;                    /* sequences, 0 .. 65535 */
  int32_t T;                    /* queries of a sequence at most */
  int32_t S;                    /* keys of a sequence at most (window attention); T with a cache */
  int32_t n_heads, n_kv_heads;  /* n_heads a multiple of n_kv_heads: query head h reads kv head h / (n_heads / n_kv_heads) */
  int32_t head_dim;             /* 64 or 128 */
  caddtree_view_t q, k, v, out; /* [B, T, n_heads, head_dim], [B, S, n_kv_heads, head_dim] twice, as q */
  float* lse;                   /* [B, T, n_heads], optional */
  const int32_t* q_len;         /* [B], optional (NULL: T).  With a tree: its nodes, n_star, to which the root is added */
  const int32_t* k_len;         /* [B], optional (NULL: S); not used with a cache */
  float scale;                  /* finite, at most 2^127 in magnitude */
  int32_t window, sinks;        /* >= 0; window 0: no window */
  caddtree_order_t order;
  caddtree_mask_t mask_kind;    /* with ORDER_TREE: U8 or BITS32, as written by caddtree_build */
  const void* mask;             /* [B, cap, cap] or [B, cap, ceil(cap / 32)] */
  const int32_t* depth;         /* [B, cap] */
  int32_t cap;                  /* of the plan that built the trees; T <= cap + 1 */
  const int32_t* page_table;    /* [B, table_pages]; the cached form only, as the next two */
  int32_t table_pages;
  const int64_t* ctx_len;       /* [B] cached tokens */
  int32_t lse_strided;          /* 0: lse is contiguous.  1, where it is read (caddtree_cache_score): element */
  int64_t lse_stride_b, lse_stride_t, lse_stride_h; /* (b, t, h) at lse + b lse_stride_b + t ..., any strides >= 0 */
} caddtree_attention_t;

/* Attention over the keys given, the queries being the last positions: query i of sequence b is at
 * position k_len - q_len + i, key j at j.  ORDER_CHAIN or ORDER_BLOCK.  Rows i >= q_len of out and lse
 * are left untouched.
 * workspace: caddtree_attention_workspace_bytes(a) bytes, 256-byte aligned, let a call with few rows
 * split its keys over the card; NULL (or fewer bytes) is accepted and keeps a row's keys in fewer parts. */
caddtree_status_t caddtree_window_attention(const caddtree_attention_t* a, void* workspace, size_t workspace_bytes,
                                            hipStream_t stream);

/* Attention over the cached keys, slots 0 .. ctx_len - 1 at positions of the same numbers, followed by
 * the new ones: key j at position ctx_len + j, in a tree at ctx_len + its depth (the root's is 0), and
 * query i where key i is.  k and v may be NULL: the queries then see the cached keys alone.  The new
 * keys are not written to the cache (caddtree_cache_write does that for those accepted). */
caddtree_status_t caddtree_cache_attention(const caddtree_cache_t* cache, const caddtree_attention_t* a,
                                           void* workspace, size_t workspace_bytes, hipStream_t stream);

/* HOST only: the workspace of the two calls above (0 where none is of use, or for sizes that they refuse). */
size_t caddtree_attention_workspace_bytes(const caddtree_attention_t* a);

/* Puts the first count[b] (NULL: T) of T new tokens of each sequence into the slots from start[b] on,
 * rounded to 4 bits.  Token j is k[b, j], or k[b, index[b, j]] where index [B, T] is given (the
 * accepted path of a tree; an index outside 0 .. rows - 1 writes nothing).  Slots past the table's end,
 * and pages outside the cache, are not written.  No two sequences may write one page's token.
 *   Rounding: E = floor(log2 m) - 2 for the largest magnitude m of a block, one more where m is above
 *   1.75 x 2^floor(log2 m) (8 is then nearer than 6); each value to the nearest code, ties to the even one. */
caddtree_status_t caddtree_cache_write(const caddtree_cache_t* cache, const caddtree_view_t* k, const caddtree_view_t* v,
                                       int32_t B, int32_t T, int32_t rows, const int64_t* start, const int32_t* count,
                                       const int32_t* index, const int32_t* page_table, int32_t table_pages,
                                       hipStream_t stream);

/* The values that slots start[b] (NULL: 0) .. end[b] - 1 stand for, at most T of them, in the cache's
 * type: slot start + j into k[b, j] and v[b, j], views that share no element (CADDTREE_E_INVALID where
 * they begin in one place).  Rows past the end, and those of pages outside the cache, are left
 * untouched. */
caddtree_status_t caddtree_cache_read(const caddtree_cache_t* cache, const caddtree_view_t* k, const caddtree_view_t* v,
                                      int32_t B, int32_t T, const int64_t* start, const int64_t* end,
                                      const int32_t* page_table, int32_t table_pages, hipStream_t stream);

/* Adds the attention weight that the cached keys get from a call's queries to their scores:
 *     new_scores[b, h, p] = scores[b, h, p] + sum_i weight[b, i] sum_g visible exp(s_igp - lse[b, i, g])
 * over the kv head's query heads g, for slots p < ctx_len; further slots are copied.  a: the arguments
 * of the caddtree_cache_attention call (q, lse as it wrote it, lengths, scale, window, sinks, order;
 * k, v, out and the mask are not used).  weight [B, T] (NULL: 1) picks and weighs queries; one at or
 * below 0 leaves its query out.  scores, new_scores [B, n_kv_heads, slots], slots >= the longest
 * ctx_len's, may be one array (else they do not overlap: CADDTREE_E_INVALID).  The order of the sums is
 * fixed. */
caddtree_status_t caddtree_cache_score(const caddtree_cache_t* cache, const caddtree_attention_t* a, const float* weight,
                                       const float* scores, float* new_scores, int64_t slots, hipStream_t stream);

/* Cuts each sequence to at most `budget` slots, by kv head: the first `sinks`, the last `recent`, and of
 * the others those with the largest scores (ties: the lower slot; a NaN counts as the lowest), in their
 * old order.  sinks + recent <= budget.  Slots of pages outside the cache hold no key and are left out,
 * sinks and recent ones among them.
 *   scores [B, n_kv_heads, slots]; new_table [B, new_pages]: pages for budget slots that are in none of
 *   the tables in use (the old pages are free once the call is done); new_scores [B, n_kv_heads,
 *   new_slots], new_slots >= budget: the kept slots' scores, then zeros; new_len [B]: how many are kept,
 *   min(ctx_len, budget) where all pages are there; kept [B, n_kv_heads, budget]: the old slots, then -1.
 *   new_scores, new_len, kept and the workspace lie in no other array of the call (scores and ctx_len
 *   among them), and new_table is not page_table: CADDTREE_E_INVALID.
 *   workspace: caddtree_evict_workspace_bytes(...) bytes, 256-byte aligned (CADDTREE_E_WORKSPACE if smaller). */
caddtree_status_t caddtree_cache_evict(const caddtree_cache_t* cache, int32_t B, const int32_t* page_table,
                                       int32_t table_pages, const int64_t* ctx_len, const float* scores, int64_t slots,
                                       int32_t budget, int32_t sinks, int32_t recent, const int32_t* new_table,
                                       int32_t new_pages, float* new_scores, int64_t new_slots, int64_t* new_len,
                                       int32_t* kept, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* HOST only: the workspace of caddtree_cache_evict (0 for rows of up to 16384 slots). */
size_t caddtree_evict_workspace_bytes(const caddtree_cache_t* cache, int32_t B, int32_t table_pages, int64_t slots);

/* ------------------------------------------------------------------------------------------------
 * Logits: what stands before and behind a tree, and what trains its drafter.
 *
 * Penalties, biases and grammar masks on the drafter's or the target's logits; the target's choice along a
 * built tree; and the loss, with its gradient, of a drafter that learns from a teacher's top logits (as
 * caddtree_reduce_topk writes them).  They take no plan; they run on the current device, with the
 * conventions at the top of this file, but for these: logits may be BF16, F16 or F32, and may be infinite
 * or NaN where a call says so.  Arithmetic is fp32 or fp64, with one rounding to the logits' type.
 *
 * Rows of V elements are strided views [B, T, V]: element (b, t, v) at data + b stride_b + t stride_t + v
 * (strides in elements, >= 0).  data is aligned to its elements; rows that start at multiples of 16 bytes
 * are somewhat faster.  An input's rows may overlap or repeat (stride 0), an output's may not.  An output
 * may be the call's logits themselves (same data and strides); else the stretches of memory from its first
 * to its last element and from the logits' first to their last do not overlap (CADDTREE_E_INVALID). */
#define CADDTREE_MAX_VOCAB (1 << 20)    /* V of these calls */
#define CADDTREE_MAX_HISTORY ((1 << 20) - 64)
#define CADDTREE_MAX_BIAS 4095
#define CADDTREE_MAX_TEACHER 256

typedef struct {
  void* data;
  int64_t stride_b, stride_t;
} caddtree_rows_t;

/* One call of caddtree_adjust_logits. */
typedef struct {
  caddtree_dtype_t dtype;
  int32_t B;                    /* sequences, 0 .. 2^19 */
  int32_t T;                    /* rows of a sequence at most; with a tree: cap + 1 */
  int32_t V;                    /* 1 .. CADDTREE_MAX_VOCAB */
  caddtree_rows_t logits, out;
  const int32_t* count;         /* [B], optional (NULL: T).  With a tree: its nodes, n_star, to which the root is added */
  const int32_t* history;       /* [B, H], optional: token ids; one outside 0 .. V - 1 is padding */
  const int32_t* history_len;   /* [B], optional (NULL: H) */
  int32_t H;                    /* 0 .. CADDTREE_MAX_HISTORY */
  const float* repetition;      /* [B] each, optional (NULL: 1, 0 and 0) */
  const float* presence;
  const float* frequency;
  const int32_t* bias_ids;      /* [B, n_bias], optional: token ids; one outside 0 .. V - 1 is padding */
  const float* bias;            /* [B, n_bias] */
  int32_t n_bias;               /* 0 .. CADDTREE_MAX_BIAS */
  const void* allowed;          /* u32 words, optional: bit (v % 32) of word v / 32 of row (b, t), which starts at word */
  int64_t allowed_stride_b;     /*   b allowed_stride_b + t allowed_stride_t (strides >= 0; 0: one mask for all) */
  int64_t allowed_stride_t;
  const int32_t* token_ids;     /* [B, T - 1] each, with a tree (else both NULL): as written by caddtree_build.  A tree of its */
  const int32_t* parent;        /*   root alone (T = 1) gives two that are not NULL, or no count */
  float fill;                   /* what a token that is not allowed gets, rounded to the logits' type (past its range: an
                                   infinity), not NaN; 0 stands for -inf.  A plan's calls take finite logits, in BF16 or
                                   F32: the drafter's get a finite one */
} caddtree_adjust_t;

/* Penalties for repeated tokens, biases and a grammar's mask.  x = the logit of token v in row (b, t), in fp32:
 *     c > 0:  x = x > 0 ? x / repetition[b] : x repetition[b];  x = x - frequency[b] c - presence[b]
 *     x = x + bias of v (of a token listed twice the last);  x = fill where v is not allowed
 * with c how often v is among the first history_len[b] tokens of history[b] and, in a tree, on the row's path:
 * the tokens of node t - 1 and of its ancestors (row 0, the root, has none; its own token belongs in the
 * history).  Of a path of more than CADDTREE_MAX_L nodes the last CADDTREE_MAX_L count; a parent that is not
 * below its node ends it.  A logit that nothing applies to is copied as it is, NaN and infinities included; one
 * that is not allowed is fill whatever it was.  A row may be left with nothing allowed: it is all fill.
 * Rows past count are left untouched.  In place (out is logits) only what changes is read and written. */
caddtree_status_t caddtree_adjust_logits(const caddtree_adjust_t* a, hipStream_t stream);

/* One call of caddtree_verify_tree. */
typedef struct {
  caddtree_dtype_t dtype;
  int32_t B;                    /* trees, 0 .. 2^19 */
  int32_t T;                    /* rows of a tree: cap + 1, the root and the nodes */
  int32_t V;                    /* 1 .. CADDTREE_MAX_VOCAB */
  caddtree_rows_t logits;       /* [B, T, V]; data NULL where `chosen` is given */
  const int32_t* chosen;        /* [B, T], optional: the target's token at each row, chosen by the caller; -1: none */
  const int32_t* token_ids;     /* [B, T - 1] each: as written by caddtree_build */
  const int32_t* parent;
  const int32_t* count;         /* [B], n_star */
  int32_t M;                    /* rows of a path at most, >= 1 */
  int32_t* accepted;            /* [B] */
  int32_t* index;               /* [B, M] */
  int32_t* tokens;              /* [B, M] */
  float* weight;                /* [B, T], optional */
} caddtree_verify_t;

/* The target's choice along a tree (Sec. 3.3).  From the root's row on: the row's token is the largest logit's (of
 * equals the lowest id; NaN and -inf are never chosen), or chosen[b, row]; if a child of the row (of several the
 * first node) carries it, the path goes on there, else it ends, as it does after M rows and where a row has no token
 * to choose.
 *   accepted[b]: rows on the path, 1 .. M;  index[b, j]: the path's rows in order, then -1;  tokens[b, j]: each
 *   one's token (-1: none), then -1.  tokens[b, accepted - 1] is the bonus token, the next tree's root.
 *   weight[b, row]: 1 on the path, else 0.
 * accepted and index are caddtree_cache_write's count and index, weight is caddtree_cache_score's.  The outputs
 * overlap nothing else.  workspace: caddtree_verify_workspace_bytes(a) bytes, 256-byte aligned, lets a call on few
 * rows read them all at once; NULL (or fewer bytes) is accepted, and the rows are read one after the other. */
caddtree_status_t caddtree_verify_tree(const caddtree_verify_t* a, void* workspace, size_t workspace_bytes, hipStream_t stream);
/* HOST only (0 where none is of use, or for sizes that the call refuses). */
size_t caddtree_verify_workspace_bytes(const caddtree_verify_t* a);

/* One call of caddtree_distill or caddtree_distill_grad. */
typedef struct {
  caddtree_dtype_t dtype;
  int32_t B;                    /* 0 .. 2^19 */
  int32_t T;
  int32_t V;                    /* 1 .. CADDTREE_MAX_VOCAB */
  caddtree_rows_t logits;       /* the student's, [B, T, V] */
  int32_t K;                    /* tokens that the teacher lists, 1 .. CADDTREE_MAX_TEACHER */
  const int32_t* ids;           /* [B, T, K]; one outside 0 .. V - 1 is padding */
  const float* target;          /* [B, T, K]: the teacher's logits, or with `tail` its log-probabilities */
  const float* weight;          /* [B, T], optional (NULL: 1) */
  float temperature;            /* finite, 2^-20 .. 2^20 */
  int32_t tail;                 /* 0 or 1 */
  float* loss;                  /* [B, T] (caddtree_distill) */
  float* stats;                 /* [B, T, 3]: optional in caddtree_distill, an input of caddtree_distill_grad */
  caddtree_rows_t grad;         /* [B, T, V] of the logits' type: optional (data NULL) in caddtree_distill */
} caddtree_distill_t;

/* Distillation from a teacher's top logits: with q = softmax(logits / temperature) of a row,
 *     p_k = exp(t_k / temperature) / sum_j exp(t_j / temperature),  rho = 0           (tail = 0)
 *     p_k = exp(t_k),  rho = max(0, 1 - sum_k p_k), the probability of all others     (tail = 1)
 *     loss = weight [ sum_k p_k (log p_k - log q_k) + rho (log rho - log(1 - Q)) ],  Q = sum of q over the listed
 *     grad_v = weight / temperature [ q_v M - (v is listed: the sum of its p_k; else: rho q_v / (1 - Q)) ]
 * with M = sum_k p_k + rho.  A term with p_k = 0 (t_k = -inf) is 0.  Where all t_k are -inf and tail = 0
 * nothing counts as listed.  The rest's mass 1 - Q is a sum of its own, at any distance from the listed tokens; its term is left
 * out where the student gives the rest nothing: where that sum, of exp((logit - largest) / temperature), is less than
 * fp64 has (2^-1074).  Padding is in no sum: with nothing listed, loss and gradient are 0.  A token listed twice
 * is two terms.  Where weight is 0 the row is not read: loss, gradient and stats are 0.  A student's logit of -inf
 * (a mask) has q = 0; in a row of nothing else every q is 0; a finite one is a logit of that value, whatever its size.  NaN and
 * +inf spread over their row.  weight / temperature has to be a number of fp32.
 *   stats[b, t]: the row's largest logit, the sum of exp((logit - largest) / temperature) (0 if all are -inf), and
 *   the same sum without the listed tokens; where that is above 0 and below 2^-126, its logarithm to base 2, a negative number.
 * caddtree_distill writes the loss and, where asked for, the gradient in one pass over the logits;
 * caddtree_distill_grad the gradient alone, from the stats that such a call kept of the same logits, ids and
 * temperature (weight: the loss's gradient).
 * The gradient may overwrite the logits.  The order of the sums is fixed by the sizes, the workspace and what is asked for.
 *   workspace: caddtree_distill_workspace_bytes(a) bytes, 256-byte aligned, lets a call of few rows split them over
 *   the card; NULL (or fewer bytes) is accepted. */
caddtree_status_t caddtree_distill(const caddtree_distill_t* a, void* workspace, size_t workspace_bytes, hipStream_t stream);
caddtree_status_t caddtree_distill_grad(const caddtree_distill_t* a, hipStream_t stream);
/* HOST only (0 where none is of use, or for sizes that the call refuses). */
size_t caddtree_distill_workspace_bytes(const caddtree_distill_t* a);

const char* caddtree_status_string(caddtree_status_t status);
const char* caddtree_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* CADDTREE_H */
