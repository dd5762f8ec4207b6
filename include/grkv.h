/*
 * grkv.h - C ABI of the MI355X (gfx950) GRKV prefill-compression path.
 *
 * GRKV ("Global Regression for KV cache", arXiv 2605.31105) compresses each
 * (layer, KV head) slice of a prefilled KV cache in two stages:
 *
 *   1. SnapKV-style span retention.  The last w prompt queries (the surrogate
 *      query window, Sec. 3.2) attend to the whole cache; every prefix token
 *      is scored by the attention it receives from the window, the scores are
 *      pooled over a window of pool_kernel neighbouring tokens, and the
 *      budget - w best prefix tokens are kept together with the w window
 *      tokens (Sec. 1 and Sec. 2, SnapKV).
 *   2. The value step of the global ridge-regression merge (Eq. 6-8;
 *      Algorithm 1, value step; App. D.1 and D.3).  With X the window's
 *      attention over the retained keys and Y its attention output over the
 *      full cache (Eq. 4), the free retained values are moved to
 *      V*_G = V0_G + X_G^T (X_G X_G^T + lambda I_m)^-1 (Y - X V0),
 *      which minimises ||Y - X V||_F^2 + lambda ||V - V0||_F^2 over V_G.
 *      Fixed tokens (sinks, the window, the top beta of the retained set,
 *      Sec. 3.4 "Fixed tokens during optimization") keep their values.
 *      Keys are not moved: K* = K0.
 *
 * A "unit" is one (layer, KV head) slice; units are independent and are
 * processed in one batched call.  G query heads share each KV head (grouped
 * query attention); their windows are stacked into m = G*w rows, row
 * r = g*w + i holding query head g at window position i, which sits at token
 * position n - w + i.
 *
 * Memory: every pointer argument is DEVICE memory owned by the caller.  The
 * library allocates nothing and keeps no state between calls; calls with
 * distinct workspaces may run concurrently on different streams.
 * Calls are asynchronous on `stream`; results are valid once the stream has
 * been synchronised.  No exception crosses this interface.
 */
#ifndef GRKV_H
#define GRKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes.  Argument errors are found on the host before anything is
 * launched, and then nothing is written. */
typedef enum {
  GRKV_OK = 0,
  GRKV_ERR_INVALID = -1,     /* bad argument (null pointer, size out of range) */
  GRKV_ERR_WORKSPACE = -2,   /* workspace smaller than grkv_workspace_bytes() */
  GRKV_ERR_UNSUPPORTED = -3, /* valid but not built: head_dim not 64/128, m = G*w > 256 */
  GRKV_ERR_HIP = -4          /* a HIP launch failed */
} grkv_status;

/* Element type of q_obs, K, V and k_out. */
typedef enum { GRKV_BF16 = 0, GRKV_F32 = 1 } grkv_dtype;

/* Per-unit status in stats[u][3]. */
#define GRKV_UNIT_OK 0
#define GRKV_UNIT_SINGULAR 1 /* non-positive Cholesky pivot: v_out holds V0 */
#define GRKV_UNIT_RANGE 2    /* internal: a window row's attention mass on the
                                retained keys is below 2^-108 of its full-cache
                                mass.  The bf16 path then redoes that unit's
                                value step against the retained set's own row
                                maxima, so a call never returns this code */

typedef struct {
  int32_t units;    /* U >= 1: number of (layer, KV head) slices */
  int32_t group;    /* G >= 1: query heads per KV head */
  int32_t head_dim; /* d: 64 or 128 */
  int32_t dtype;    /* grkv_dtype */
} grkv_problem;

/* Fixed-token and masking options.  NULL selects the defaults
 * {n_sink = 4, beta = 0.10f, fix_window = 1, causal_window = 1}:
 * the paper keeps sink tokens, the window tokens and the top 10% retained
 * tokens fixed (Sec. 4.1 hyperparameters). */
typedef struct {
  int32_t n_sink;        /* retained positions below n_sink stay fixed (>= 0) */
  float beta;            /* in [0, 1]: the first floor(beta * budget) prefix
                            tokens of the selection order stay fixed */
  int32_t fix_window;    /* nonzero: the w window tokens stay fixed */
  int32_t causal_window; /* nonzero: window row at position p sees keys 0..p only */
} grkv_options;

/* Outputs, all device memory owned by the caller, c = budget:
 *   idx   int32 [U][c]      retained positions, ascending; the last w entries
 *                           are n-w .. n-1.  Ties in the pooled score go to the
 *                           lower position.
 *   k_out dtype [U][c][d]   K0 = K[idx], bit-exact copies of the input rows
 *   v_out float [U][c][d]   merged values V*
 *   stats float [U][4]      {||Y||_F^2, D_before, D_after, unit status}, where
 *                           D = ||Y - X V||_F^2 / ||Y||_F^2 (the raw numerator
 *                           when ||Y|| = 0) with V = V0 and V = V*; may be NULL
 *   workspace               at least grkv_workspace_bytes() bytes, 256-byte
 *                           aligned; its contents on return are described by
 *                           grkv_workspace_layout(). */
typedef struct {
  int32_t* idx;
  void* k_out;
  float* v_out;
  float* stats;
  void* workspace;
  size_t workspace_bytes;
  /* Optional timing hooks, may be NULL: an array of 2 * GRKV_NUM_STAGES
   * hipEvent_t owned by the caller.  For every stage s whose two slots are both
   * non-null, slot 2s is recorded on `stream` before the stage's kernels and
   * slot 2s+1 after them, so hipEventElapsedTime gives the stage's duration. */
  void** stage_events;
} grkv_outputs;

/* Stages of one call, in launch order (indices into stage_events / 2).  A stage
 * that a given call does not run leaves its two events unrecorded: the bf16
 * path (head_dim 64/128, G*w <= 128) folds FULL_Y, RESID and GRAM into
 * neighbouring stages, reads the retained rows inside RET_PROB (no GATHER) and
 * forms the retained softmax from the full-cache log-sum-exp (no RET_LSE).  fp32
 * calls of up to 128 rows record every stage but KEY; their RESID follows GRAM
 * and holds the sums of the X V0 and N partials (nothing in calls of one or two
 * of them each), R itself is formed in SOLVE. */
enum {
  GRKV_STAGE_FULL_LSE = 0,     /* full-cache pass A: reference / sum-exp per split */
  GRKV_STAGE_FULL_LSE_COMBINE, /* -> log-sum-exp of every window row */
  GRKV_STAGE_FULL_PROB,        /* full-cache pass B: P.V partials, SnapKV column sums */
  GRKV_STAGE_FULL_Y,           /* -> Y */
  GRKV_STAGE_SELECT,           /* pooling, top-k, fixed set */
  GRKV_STAGE_GATHER,           /* K0 -> k_out, V0 (generic path) */
  GRKV_STAGE_RET_LSE,          /* retained-cache pass A (generic path) */
  GRKV_STAGE_RET_LSE_COMBINE,
  GRKV_STAGE_RET_PROB,         /* retained-cache pass B: X V0 (and on the bf16 path
                                  K0 -> k_out, Gram and retained-mass partials) */
  GRKV_STAGE_RESID,            /* R = Y - X V0, or the sums it is formed from */
  GRKV_STAGE_GRAM,             /* N partials */
  GRKV_STAGE_SOLVE,            /* (Y, R, N combines,) Cholesky, Z, stats */
  GRKV_STAGE_UPDATE,           /* V* = V0 + X_G^T Z */
  GRKV_STAGE_KEY,              /* key step (grkv_compress_kv only): CG, K* */
  GRKV_NUM_STAGES
};

/* Compress U units.
 *   q_obs  dtype [U][G][w][d]  the window queries (post-RoPE), query head
 *                               kv_head*G + g of unit u at [u][g]
 *   K, V   dtype [U][n][d]     the full cache (post-RoPE keys)
 *   n            tokens per unit, w <= budget <= n, n <= 2^30
 *   window       w >= 1
 *   budget       c: retained tokens including the w window tokens
 *   pool_kernel  odd k >= 1: scores are summed over positions j-(k-1)/2 ..
 *                j+(k-1)/2 (zero outside the prefix) before ranking
 *   lambda       ridge coefficient lambda_v >= 0 (finite)
 *   stream       hipStream_t, NULL for the default stream
 * Errors: GRKV_ERR_INVALID for null pointers, units < 1, group < 1,
 * window < 1, budget < window, budget > n, even or < 1 pool_kernel,
 * negative or non-finite lambda, beta outside [0, 1], n_sink < 0, an unknown
 * dtype; GRKV_ERR_UNSUPPORTED for head_dim not in {64, 128} or G*w > 256;
 * GRKV_ERR_WORKSPACE when out->workspace_bytes is too small; GRKV_ERR_HIP
 * when a launch fails (outputs are then undefined). */
int grkv_compress(const void* q_obs, const void* K, const void* V, int64_t n,
                  int32_t window, int32_t budget, int32_t pool_kernel,
                  float lambda, void* stream, const grkv_problem* prob,
                  const grkv_options* opt, const grkv_outputs* out);

/* grkv_compress for callers that cannot allocate device memory (code under
 * stream capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same computation, kernels and arguments, but the workspace is a device array
 * of GRKV_NOALLOC_SCRATCH_BYTES held by the library on every device it runs on
 * (until the process ends); out->workspace and out->workspace_bytes are not
 * read.  The call runs on the current device (stream must belong to it) and
 * calls no allocating routine.  The first call on a device looks up the
 * array's address there.  Every call on one device shares that array: calls
 * that overlap on one device (several streams or host threads) race on it.
 * Nothing in it needs to start at zero.  Errors: those of grkv_compress;
 * GRKV_ERR_WORKSPACE when grkv_workspace_bytes() for the shape exceeds
 * GRKV_NOALLOC_SCRATCH_BYTES (64 MiB holds, for example, a one-layer call of
 * 8 KV heads, n = 32768, w = 32, budget 2048, d = 128: 54.5 MiB). */
#define GRKV_NOALLOC_SCRATCH_BYTES (64ull << 20)
int grkv_compress_noalloc(const void* q_obs, const void* K, const void* V, int64_t n,
                          int32_t window, int32_t budget, int32_t pool_kernel,
                          float lambda, void* stream, const grkv_problem* prob,
                          const grkv_options* opt, const grkv_outputs* out);

/* Key step of GRKV (Sec. 3.4 "Key step" and "Linearized dual solution",
 * Eq. 9-10; Algorithm 1, key step; App. D.2 and D.3), run by grkv_compress_kv
 * after the value step with the merged values V* held fixed and the keys at K0
 * (one alternating step, S = 1, the paper's default).  With f(K) =
 * softmax(Q K^T / sqrt(d)) V* over the retained keys, E = Y - f(K0) and J_G the
 * derivative of f with respect to the free keys, the free keys move to
 *   K*_G = K0_G + unvec(J_G^T alpha),
 *   alpha = (J_G J_G^T + lambda_k I_{md})^-1 vec(E),
 * which minimises ||E - J_G dK||^2 + lambda_k ||dK||^2; fixed keys keep K0.
 * The md x md system is solved matrix-free by conjugate gradients from
 * alpha = 0.  NULL options select {lambda_k = lambda, max_iter = 64,
 * tol = 1e-5f, steps = 1} (the paper uses lambda_k = lambda_v and does not
 * state its CG settings). */
typedef struct {
  float lambda_k;   /* ridge coefficient of the keys, >= 0 and finite */
  int32_t max_iter; /* conjugate-gradient iterations at most, 0 .. 4096 */
  float tol;        /* stop once ||r|| <= tol ||rhs|| (recursive residual), >= 0 */
  int32_t steps;    /* alternating value/key steps S, 1 .. 16 (Algorithm 1; the
                       paper's default and best setting is 1).  Step t > 1 takes
                       the value step at the current keys K^(t) (X from K^(t),
                       the update still anchored at V0) and the key step
                       linearized at K^(t), whose right-hand side gains
                       J_G (K^(t) - K0).  All S steps run (the paper's early
                       stop at a change <= 1e-9 is below fp32 resolution). */
} grkv_key_options;

/* Per-unit key-step outcome in cg_info[u][2]. */
#define GRKV_KEY_CONVERGED 1 /* the residual reached tol */
#define GRKV_KEY_MAX_ITER 2  /* max_iter iterations ran first */
#define GRKV_KEY_SKIPPED 3   /* the unit's value step reported a non-zero
                                status (stats[u][3]): K* = K0 */
#define GRKV_KEY_BREAKDOWN 4 /* a CG step found p^T A p <= 0 (possible only
                                for lambda_k = 0); the last iterate is kept */

/* grkv_compress followed by the key step (and, for steps > 1, further
 * alternating value and key steps).  All arguments as for grkv_compress; in
 * addition
 *   kopt     key-step options, or NULL for the defaults above
 *   k_star   float [U][c][d]   merged keys K*, device memory (required);
 *                              k_out still receives K0
 *   cg_info  float [U][4]      of the last key step: {CG iterations, final
 *                              ||r|| / ||rhs||, GRKV_KEY_* outcome, ||rhs||_F},
 *                              or NULL
 * v_out and stats hold the last value step.  out->workspace_bytes must be at
 * least grkv_workspace_bytes_kv() for the same number of steps.
 * Errors: those of grkv_compress; GRKV_ERR_INVALID for a null k_star or bad
 * kopt; GRKV_ERR_UNSUPPORTED unless dtype is bf16 and G*w <= 128. */
int grkv_compress_kv(const void* q_obs, const void* K, const void* V, int64_t n,
                     int32_t window, int32_t budget, int32_t pool_kernel,
                     float lambda, void* stream, const grkv_problem* prob,
                     const grkv_options* opt, const grkv_outputs* out,
                     const grkv_key_options* kopt, float* k_star, float* cg_info);

/* Workspace bytes grkv_compress_kv needs for `steps` alternating steps; 0 if
 * invalid or unsupported. */
size_t grkv_workspace_bytes_kv(const grkv_problem* prob, int64_t n,
                               int32_t window, int32_t budget, int32_t steps);

/* The default key options for a value ridge coefficient lambda. */
void grkv_default_key_options(grkv_key_options* kopt, float lambda);

/* Per-unit (ragged) budgets: the back-ends the paper pairs GRKV with (Sec. 4,
 * compatibility) differ in how much of the cache each unit keeps (PyramidKV
 * per layer, Ada-KV per head); the merge is unchanged.  grkv_compress_ragged
 * compresses unit u exactly as grkv_compress would with budget budgets[u]
 * (w <= budgets[u] <= n; the fixed set uses floor(beta * budgets[u])).
 *   budgets  int32 [U], HOST memory
 *   out      packed outputs: idx int32 [sum c_u], k_out dtype [sum c_u][d],
 *            v_out float [sum c_u][d], unit u starting at slot
 *            off_u = budgets[0] + ... + budgets[u-1]; stats [U][4] as before
 * On the bf16 path (d 64/128, group * window <= 128) every stage is one launch
 * over all units: a per-unit table (slot offset, budget, splits) is copied
 * into the workspace from host memory on `stream` first (the host array may
 * be reused once the call returns; a copy from pageable memory, so the call
 * is not for HIP graph capture), and out->stage_events is honoured as for
 * grkv_compress.  Other shapes run consecutive units of equal budget as one
 * grkv_compress batch each (out->stage_events ignored).  The workspace is
 * grkv_workspace_bytes_ragged(); errors as for grkv_compress, and
 * GRKV_ERR_UNSUPPORTED when the budgets sum past 2^31 - 1. */
int grkv_compress_ragged(const void* q_obs, const void* K, const void* V, int64_t n,
                         int32_t window, const int32_t* budgets, int32_t pool_kernel,
                         float lambda, void* stream, const grkv_problem* prob,
                         const grkv_options* opt, const grkv_outputs* out);

size_t grkv_workspace_bytes_ragged(const grkv_problem* prob, int64_t n, int32_t window,
                                   const int32_t* budgets);

/* Pyramid schedule (PyramidKV: lower layers keep more of the cache, higher
 * layers less): budgets fall linearly from (2 - ratio) * mean_budget at layer
 * 0 to ratio * mean_budget at the top layer, rounded to nearest, clipped to
 * [window, n], with the rounding remainder given to the lowest layers so that
 * the layers' mean stays mean_budget where the clip allows.  Every head of a
 * layer gets the layer's budget; units are layer-major (u = layer * kv_heads
 * + head).  budgets: int32 [layers * kv_heads], HOST memory.  ratio in [0, 1];
 * errors: GRKV_ERR_INVALID. */
int grkv_pyramid_budgets(int32_t layers, int32_t kv_heads, int32_t mean_budget, int32_t window,
                         int64_t n, float ratio, int32_t* budgets);

/* Adaptive per-head budgets (Ada-KV: heads that need long-range context keep
 * more): inside each layer the kv_heads heads share kv_heads * (budget - w)
 * selected tokens, taken as the highest pooled scores over all its heads (ties
 * to the lower head, then the lower position); head h gets w plus the number
 * of its tokens taken.  pooled: float [U][n - w] device memory, the pooled
 * scores of a grkv_compress call (grkv_workspace_layout().pooled); budgets:
 * int32 [U] device memory, written asynchronously on stream.  kv_heads <= 128.
 * The scores must be finite and non-negative (pooled attention masses are);
 * one block per layer selects by radix over their bit patterns.
 * Errors: GRKV_ERR_INVALID, GRKV_ERR_UNSUPPORTED, GRKV_ERR_HIP. */
int grkv_adaptive_budgets(const float* pooled, int32_t layers, int32_t kv_heads, int64_t n,
                          int32_t window, int32_t budget, void* stream, int32_t* budgets);

/* Token scores of H2O (Sec. 2: heavy-hitter tokens kept by accumulated
 * attention scores; Sec. 4.3, compatibility), the token-based eviction
 * back-end GRKV is paired with.  For unit u the score of prefix token j < n - w
 * is the attention it receives summed over every prompt position i >= j of
 * every query head g of the unit's group, each row being the causal softmax of
 * q_{g,i} . k / sqrt(d) over keys 0..i:
 *   s_j = sum_g sum_{i >= j} exp(q_{g,i} . k_j / sqrt(d) - LSE_{g,i}).
 *   q_all    dtype [U][G][n][d]  the queries of every prompt position (post-RoPE)
 *   K        dtype [U][n][d]
 *   scores   float [U][n - w]    out (device memory)
 *   workspace                    >= grkv_h2o_workspace_bytes(), 256-byte aligned
 * bf16 only, head_dim 64 or 128, group 1, 2, 4 or 8.  The cost is that of a
 * prefill attention without P.V (two passes of O(n^2 d) MFMA work per head).
 * Errors: GRKV_ERR_INVALID (null pointers, window outside [1, n], bad sizes),
 * GRKV_ERR_UNSUPPORTED, GRKV_ERR_WORKSPACE, GRKV_ERR_HIP.  Asynchronous on
 * stream; allocates nothing. */
int grkv_h2o_scores(const void* q_all, const void* K, int64_t n, int32_t window, void* stream,
                    const grkv_problem* prob, float* scores, void* workspace,
                    size_t workspace_bytes);

/* Workspace bytes of grkv_h2o_scores (the row log-sum-exps, U * G * n floats);
 * 0 if the shape is invalid or unsupported. */
size_t grkv_h2o_workspace_bytes(const grkv_problem* prob, int64_t n);

/* grkv_compress with the selection driven by caller-supplied per-token scores
 * instead of the window attention's column sums: the form a token-based
 * eviction front-end such as H2O (scores from grkv_h2o_scores, pool_kernel 1)
 * takes.  scores: float [U][n - w] device memory, finite and non-negative
 * (attention masses are), pooled with pool_kernel exactly as the column sums
 * would be; the top floor(beta * c) fixed subset follows the same order.  The
 * window attention, Y and the value step are those of grkv_compress.  All
 * other arguments, outputs, workspace and errors as for grkv_compress
 * (GRKV_ERR_INVALID also for a null scores when n > window). */
int grkv_compress_scored(const void* q_obs, const void* K, const void* V, int64_t n,
                         int32_t window, int32_t budget, int32_t pool_kernel, float lambda,
                         void* stream, const grkv_problem* prob, const grkv_options* opt,
                         const float* scores, const grkv_outputs* out);

/* Carrier concentration of a local merge rule (App. B, "Quantitative Carrier
 * Concentration"; Sec. 1): the diagnostic the paper uses to show that, after
 * span-based eviction, a key-similarity matcher (as in D2O/KVMerger) loads a
 * few span-boundary tokens with most of the evicted tokens.  Every evicted
 * token j is assigned to the retained slot i with the highest key cosine
 * similarity cos(k_j, k_idx[i]) over all retained tokens (equal values go to
 * the lower slot; a zero key has cosine 0 with all), and with a_i the number of
 * tokens assigned to slot i:
 *   K        dtype [U][n][d]  the full cache keys (bf16 only)
 *   idx      int32 [U][c]     ascending retained positions (grkv_compress)
 *   stats    float [U][4]     the stats of a grkv_compress call, or NULL
 *   assign   int32 [U][n]     out: slot of each evicted position, -1 for the
 *                             retained positions (required)
 *   counts   int32 [U][c]     out: a_i, or NULL
 *   metrics  float [U][8]     out: {b = #(a_i > 0), b_eff = (sum a)^2 / sum a^2,
 *                             A_max = max a / mean a, Gini of the a_i (mean
 *                             absolute difference over all pairs / twice the
 *                             mean), boundary fraction (first and last slots
 *                             of each run of consecutive positions, over c),
 *                             boundary share of the assignments, enrichment
 *                             (share / fraction), boundary / interior mean
 *                             load (NaN without both kinds; the load figures
 *                             are NaN when nothing is evicted)}
 *   l_common float [1]        out (needs stats): the discrepancy summed over the
 *                             units, sum D_after ||Y||^2 / sum ||Y||^2 (the
 *                             paper's L_common over these units), or NULL
 * Errors: GRKV_ERR_INVALID for null required pointers, units or group < 1, an
 * unknown dtype, budget outside [1, n]; GRKV_ERR_UNSUPPORTED for fp32 keys, d
 * not 64/128 or budget > 8192; GRKV_ERR_HIP for a failed launch.  Allocates
 * nothing; asynchronous on stream. */
int grkv_carrier_stats(const void* K, int64_t n, int32_t budget, const grkv_problem* prob,
                       const int32_t* idx, const float* stats, void* stream, int32_t* assign,
                       int32_t* counts, float* metrics, float* l_common);

/* ------------------------------------------------------------------------
 * Pages of a cache.  What a call above returns (retained keys, merged values)
 * is kept, grown by new tokens, branched and thinned in the pages of one pool.
 * A unit of the pool is one (sequence, layer, KV head) slice of any length L:
 * its slot s (0 <= s < L) lies in page table[u][s / page_size], row
 * s % page_size, so units with budgets of their own share one pool.  All memory
 * is the caller's:
 *   k, v       dtype [pages][page_size][head_dim], 16-byte aligned
 *   table      int32 [units][max_pages]: the pages of each unit in slot order,
 *              -1 behind them
 *   lens       int32 [units]: L
 *   refs       int32 [pages]: how many tables hold each page
 *   free_bits  uint32 [ceil(pages / 32)]: bit p % 32 of word p / 32 is set where
 *              page p is in no table (refs[p] = 0)
 * page_size is a power of two, 16 .. 1024.  table .. free_bits are the calls' to
 * write (after grkv_pages_init); a page that is not full is in one table only,
 * which every call keeps so.  New pages are the free ones of lowest number,
 * handed out in the order of the entries and of the slots of each entry, so a
 * pool's state never depends on timing. */
typedef struct {
  void* k;
  void* v;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  uint32_t* free_bits;
  int32_t pages, page_size, units, max_pages;
  int32_t head_dim; /* 64 or 128 */
  int32_t dtype;    /* grkv_dtype of k and v */
} grkv_pages;

/* Outcome of one entry of a call on pages, in status[i]. */
#define GRKV_PAGES_OK 0
#define GRKV_PAGES_FULL 1   /* too few free pages for this entry and those before it */
#define GRKV_PAGES_LENGTH 2 /* more rows than the unit's table row holds */
#define GRKV_PAGES_UNIT 3   /* no such unit; the unit is written by an earlier entry of
                               the call, or read here and written by another entry; or
                               the destination of a copy is another unit and not empty */
#define GRKV_PAGES_RANGE 4  /* rows outside their source */

/* The units a call works on, one per entry: device arrays of `entries`
 * elements.  An entry with a status other than GRKV_PAGES_OK leaves its unit as
 * it was (one exception: grkv_pages_compact); the others go ahead. */
typedef struct {
  int32_t entries;       /* >= 0; with 0 a call does nothing */
  const int32_t* units;  /* unit of each entry, or NULL: entry i is unit i */
  int32_t rows;          /* rows per entry (the largest, with counts) */
  const int32_t* counts; /* rows of each entry, taken to 0 .. rows; NULL: rows each */
  const int64_t* starts; /* first row of each entry in the packed source of
                            source_rows rows; NULL: i * rows */
  int64_t source_rows;
  int32_t* status;       /* out [entries], or NULL */
} grkv_page_entries;

/* An empty pool: no unit holds a row, every page is free. */
int grkv_pages_init(const grkv_pages* pages, void* stream);

/* Appends rows to units: row j of entry i, at slot lens[u] + j, is row
 * starts[i] + j of k and v [source_rows][head_dim], which have types of their
 * own (k_out is bf16 beside a float v_out) and are rounded to the pool's, to
 * nearest even.  k and v are 16-byte aligned and not part of the pool.  A unit
 * may be in a call once. */
int grkv_pages_append(const grkv_pages* pages, const grkv_page_entries* entries, const void* k,
                      int32_t k_dtype, const void* v, int32_t v_dtype, void* stream,
                      void* workspace, size_t workspace_bytes);

/* Unit dst[i] (int32 [entries], device memory; empty before) becomes a copy of
 * unit units[i]: the full pages are shared, the rows of a last page that is not
 * full are copied to one of its own.  A unit may be the source of many entries; one
 * that is its own destination (dst[i] equal to units[i]) stays as it is, GRKV_PAGES_OK.
 * rows, counts, starts and source_rows are not read. */
int grkv_pages_fork(const grkv_pages* pages, const grkv_page_entries* entries, const int32_t* dst,
                    void* stream, void* workspace, size_t workspace_bytes);

/* The rows of a unit that are to stay: unit dst[i] becomes slots 0 .. keep[i] - 1
 * of unit units[i], then its slots idx[starts[i]] .. idx[starts[i] + counts[i] - 1]
 * (int32 [source_rows], any order, repeats allowed).  dst NULL: in place (the pages
 * that a unit no longer needs are free after the call); else dst[i] is empty before or
 * equals units[i].  keep NULL: 0.  idx may be NULL where rows is 0 (a cache taken
 * back to its first keep[i] slots).  The full pages under keep[i] are shared, or
 * stay in place; the rows behind them go to new pages, which are taken before the
 * old ones are given up; only slots taken back in place keep a last page that is
 * not shared.  keep[i] outside 0 .. L gives GRKV_PAGES_RANGE; an index outside
 * 0 .. L - 1 too, but then the entry is carried out with a row of zeros there. */
int grkv_pages_compact(const grkv_pages* pages, const grkv_page_entries* entries,
                       const int32_t* dst, const int32_t* keep, const int32_t* idx, void* stream,
                       void* workspace, size_t workspace_bytes);

/* Units give up their rows; a page that no table holds any more is free.  A unit
 * named twice is freed once; GRKV_PAGES_UNIT is the only status. */
int grkv_pages_free(const grkv_pages* pages, const grkv_page_entries* entries, void* stream);

/* Workspace bytes of grkv_pages_append, _fork and _compact for this many
 * entries, 256-byte aligned; 0 if invalid. */
size_t grkv_pages_workspace_bytes(const grkv_pages* pages, int32_t entries);

/* All of these are asynchronous on stream, allocate nothing and may be captured.
 * Errors: GRKV_ERR_INVALID for null pointers, misaligned k, v or workspace, sizes out of
 * range (pages, units, max_pages < 1, pages > 2^30, max_pages * page_size > 2^30, entries or
 * rows < 0, entries * (rows + page_size) >= 2^31, 2^24 entries or more of a fork, a compaction
 * or a free), an unknown dtype;
 * GRKV_ERR_UNSUPPORTED for another head_dim or page_size;
 * GRKV_ERR_WORKSPACE; GRKV_ERR_HIP. */

/* Attention over pages: single tokens, or trees of drafted tokens.  Entry e is a
 * unit of the pool whose last t slots (t = tokens, or counts[e]) are drafted
 * tokens, stored there by grkv_pages_append; query i of each of the `group`
 * heads is the i-th of them.  Token i follows drafted token parents[i] < i, or the
 * cache itself (-1).  It lies at position L - t + depth (depth: its number of
 * drafted ancestors) and sees the slots j < L - t before the drafted ones, itself
 * and its ancestors, of these with window > 0 only positions below n_sink or the
 * last `window` up to its own (slot j < L - t is position j):
 *   o = sum_j softmax_j(q . k_j / sqrt(d)) v_j,  lse = ln sum_j exp(q . k_j / sqrt(d)).
 * A query that sees nothing (or whose weights are all zero) gets o = 0, lse =
 * -infinity.  What a query does not see never reaches it, infinities and NaN
 * included (its last bits may differ beside those, as its rows are summed in another way). */
typedef struct {
  int32_t entries;        /* >= 0; with 0 the call does nothing */
  int32_t group;          /* query heads per KV head, >= 1 */
  int32_t tokens;         /* queries per head, 1 .. 64 */
  const int32_t* units;   /* int32 [entries]: unit of each entry, or NULL: entry e is
                             unit e.  An entry whose unit is not in the pool sees nothing */
  const int32_t* counts;  /* int32 [entries]: drafted tokens of each entry, taken to
                             0 .. tokens; o and lse of queries from counts[e] on stay as
                             they were.  NULL: tokens each */
  const int32_t* parents; /* int32 [trees][tokens], or NULL: a chain (each token follows
                             the one before).  Parents outside -1 .. i - 1 count as -1 */
  int32_t trees;          /* trees: entries e of equal e / (entries / trees) have one tree;
                             divides entries (not read without parents) */
  int32_t window;         /* >= 0; 0: none */
  int32_t n_sink;         /* >= 0 (not read without a window) */
} grkv_tree;

/* q, o: pages' dtype [entries][group][tokens][head_dim], 16-byte aligned; lse float
 * [entries][group][tokens] or NULL; neither may overlap q, the pool or another array of the
 * call.  Over bf16 values a weight is held to 2^-15 of it where memory bounds a call (up to 64
 * rows, group * tokens, a unit, and small calls of more) and rounded to bf16 (2^-8) in the others;
 * sums are float32, of weights of 1 at most.  The length of a unit is read on the device.  Errors:
 * those of the calls on pages; GRKV_ERR_INVALID for bad counts in `tree` (also
 * entries * group * tokens * head_dim >= 2^40, and 2^24 blocks or more: entries times the row
 * groups of a unit, of 16 rows at least); GRKV_ERR_UNSUPPORTED for tokens > 64. */
int grkv_tree_attention(const void* q, const grkv_pages* pages, const grkv_tree* tree, void* o,
                        float* lse, void* stream, void* workspace, size_t workspace_bytes);

size_t grkv_tree_attention_workspace_bytes(const grkv_pages* pages, const grkv_tree* tree);

/* Causal attention with a sliding window and sink tokens over contiguous keys:
 * query i of nq is position p = n - nq + i (a whole prompt with nq = n, a chunk of
 * one, a single token) and sees keys j <= p with j > p - window or j < n_sink;
 * window 0: all j <= p.
 *   q, o     dtype [U][G][nq][d]
 *   K, V     dtype [U][n][d]
 *   lse      float [U][G][nq], or NULL
 * all 16-byte aligned; o and lse as in grkv_tree_attention.  Errors:
 * GRKV_ERR_INVALID (null pointers, nq outside 1 .. n, n > 2^30, window or n_sink
 * < 0, units or group < 1, an unknown dtype, U * G * nq * d >= 2^40, 2^24 blocks or
 * more as above), GRKV_ERR_UNSUPPORTED (head_dim), GRKV_ERR_WORKSPACE, GRKV_ERR_HIP. */
int grkv_sink_attention(const void* q, const void* K, const void* V, int64_t n, int32_t nq,
                        int32_t window, int32_t n_sink, void* stream, const grkv_problem* prob,
                        void* o, float* lse, void* workspace, size_t workspace_bytes);

size_t grkv_sink_attention_workspace_bytes(const grkv_problem* prob, int64_t n, int32_t nq,
                                           int32_t window, int32_t n_sink);

/* ------------------------------------------------------------------------
 * A step of a served model over pages.  A step takes new tokens of a batch of
 * sequences, any number of each (a token where a sequence decodes, a chunk of its
 * prompt, or none), packed one behind the other into `tokens` rows; sequence b's
 * rows are starts[b] .. starts[b + 1] - 1.  Each sequence has `heads` units of a
 * pool, of lengths of their own: those of a layer's KV heads, or of all layers'
 * (then one grkv_pages_extend serves the whole step).  A layer of the step is
 *   grkv_pages_extend    the units grow; every token's position and slots,
 *   grkv_pages_store     queries and keys rotated, keys and values stored there,
 *   grkv_chunk_attention attention of the new tokens over their units. */
typedef struct {
  int32_t sequences;    /* >= 0; with 0 a call does nothing */
  int32_t heads;        /* units of a sequence, >= 1 */
  const int32_t* units; /* int32 [sequences][unit_stride]: the unit of head h of sequence b at
                           b * unit_stride + h; NULL: unit b * heads + h */
  int64_t unit_stride;  /* >= heads (not read without units) */
  int32_t tokens;       /* rows of the packed tokens, >= 0 */
} grkv_step;

/* Of rows that are no sequence's, or a refused one's: they have no position. */
#define GRKV_NO_POSITION INT32_MIN

/* Grows the units of every sequence by counts[b] (int32 [sequences], below 0 taken as 0)
 * rows, whose content is whatever the pages held, and gives
 *   starts     int32 [sequences + 1]    sums of the counts before each sequence, `tokens` at most
 *   positions  int32 [tokens]           seen[b] + i of the i-th new token of sequence b
 *   slots      int64 [tokens][heads]    where row lens[u] + i of its units is to be stored:
 *                                       row page * page_size + s % page_size of k and v
 *   status     int32 [sequences]        or NULL
 * seen (int32 [sequences]): how many tokens a sequence had, which its units' lengths do not say
 * once they are compressed; NULL: the length of its first unit.  All units of a sequence
 * grow, or none: a sequence is refused for the largest of its units' GRKV_PAGES_ codes (_UNIT
 * also for a unit that an earlier head or sequence of the call names; _RANGE: it has new tokens
 * and their rows pass `tokens`, seen[b] is below 0, or what it has seen after the call, seen[b] +
 * counts[b], passes 2^31 - 1), and its rows, like those behind the last sequence, have position
 * GRKV_NO_POSITION and slots -1.  New pages are handed out in the order of the sequences and their
 * heads. */
int grkv_pages_extend(const grkv_pages* pages, const grkv_step* step, const int32_t* counts,
                      const int32_t* seen, int32_t* starts, int32_t* positions, int64_t* slots,
                      int32_t* status, void* stream, void* workspace, size_t workspace_bytes);

/* 256-byte aligned; 0 if invalid. */
size_t grkv_pages_extend_workspace_bytes(const grkv_pages* pages, const grkv_step* step);

/* Rotary positions: the first `dims` columns of a row are dims / 2 pairs (a, b), columns
 * (2 i, 2 i + 1) where interleaved, else (i, i + dims / 2); at position p pair i becomes
 *   scale * (a cos x - b sin x, a sin x + b cos x),  x = p freqs[i],
 * or with `inverse` the same with -x, which carries a gradient back through the call.  Angles
 * are formed in 64 bits; the other columns stay as they are. */
typedef struct {
  const double* freqs;  /* [dims / 2], device memory: radians per position */
  int32_t dims;         /* even, 2 .. head_dim */
  int32_t interleaved;
  int32_t inverse;
  float scale;
} grkv_rotation;

/* Rows of heads: column c of head h of token t at data[t * token_stride + h * head_stride + c]
 * (strides in elements, any layout with whole rows). */
typedef struct {
  void* data;
  int64_t token_stride, head_stride;
} grkv_rows;

/* y = x rotated: `heads` rows of head_dim columns for each of `tokens` tokens at positions
 * int32 [tokens] (any sign; rows of a token at GRKV_NO_POSITION are left as they were).  y is x
 * itself (data and strides) or does not overlap it.  Float32 inside, rounded once.  Rows
 * whose addresses and parts are multiples of 16 bytes take the fast path. */
int grkv_rotary(const grkv_rows* x, const grkv_rows* y, int32_t tokens, int32_t heads,
                int32_t head_dim, int32_t dtype, const int32_t* positions,
                const grkv_rotation* rotation, void* stream);

/* Host only: the frequencies of base^(-2 i / dims) radians, scaled for contexts `factor` (>= 1)
 * times as long as the `length` that a model was trained at, into freqs [dims / 2] (host memory):
 *   GRKV_ROTARY_PLAIN   as they are
 *   GRKV_ROTARY_LINEAR  divided by factor
 *   GRKV_ROTARY_BASE    of base * factor^(dims / (dims - 2)): the lowest divided by factor (2 dims:
 *                       as they are)
 *   GRKV_ROTARY_PARTS   f (1 - y + y factor) / factor with y = (length f / (2 pi) - low) / (high - low)
 *                       taken to 0 .. 1: pairs that make `high` turns or more over the length
 *                       stay, those of `low` or fewer are divided (arXiv 2309.00071, Sec. 3.2)
 * GRKV_ERR_INVALID for constants that are not finite, a base, factor or length not above zero, a
 * factor below 1, low < 0 or high <= low (each where the method reads it), and where the scaled base or
 * a frequency passes 64 bits or falls to zero; freqs then means nothing. */
#define GRKV_ROTARY_PLAIN 0
#define GRKV_ROTARY_LINEAR 1
#define GRKV_ROTARY_BASE 2
#define GRKV_ROTARY_PARTS 3
int grkv_rotary_freqs(int32_t dims, double base, int32_t method, double factor, double length,
                      double low, double high, double* freqs);

/* Stores the step's keys and values: row (t, h) of k and v goes to row slots[t * slot_stride + h]
 * of the pool's k and v, rounded to the pool's type; a negative slot, or one past the pool's
 * rows, stores nothing.  With a rotation keys are rotated by positions, and so are q's `q_heads`
 * rows into q_out (as in grkv_rotary); rows of tokens at GRKV_NO_POSITION are left as they were.
 * rotation NULL: positions and q are not read.  q_heads 0: no queries.  k, v and q have head_dim
 * columns of one type, dtype.  q_out overlaps neither k and v nor the pool.  Slots of a call are
 * different from one another (grkv_pages_extend's are). */
int grkv_pages_store(const grkv_pages* pages, int32_t tokens, int32_t heads, const int64_t* slots,
                     int64_t slot_stride, const grkv_rows* k, const grkv_rows* v, int32_t dtype,
                     const grkv_rows* q, const grkv_rows* q_out, int32_t q_heads,
                     const int32_t* positions, const grkv_rotation* rotation, void* stream);

/* Attention of the new tokens: the c = starts[b + 1] - starts[b] (`longest` at most) tokens of
 * sequence b are the last c slots of each of its units, query head h * group + g reads
 * the unit of head h, and query i sees the slots j <= p = L - c + i, with window > 0 only
 * j > p - window or j < n_sink:
 *   q, o  pages' dtype [tokens][heads * group][head_dim], 16-byte aligned
 *   lse   float [tokens][heads * group], or NULL
 * as in grkv_tree_attention, also for queries that see nothing and for values that are not
 * seen.  Over bf16 values weights are held to 2^-15 of them for a sequence's rows (tokens times
 * group) up to 64, and for the last 64 or fewer past a multiple of 128; the others are rounded to bf16
 * (2^-8).  Rows of no sequence, and those from a sequence's `longest` on, stay as they were.
 * `longest` bounds the workspace.  Of a refused sequence (grkv_pages_extend) the rows mean nothing. */
typedef struct {
  int32_t group;    /* query heads per unit, >= 1 */
  int32_t longest;  /* most new tokens of a sequence, >= 1 */
  int32_t window;   /* >= 0; 0: none */
  int32_t n_sink;   /* >= 0 (not read without a window) */
} grkv_chunk;

int grkv_chunk_attention(const void* q, const grkv_pages* pages, const grkv_step* step,
                         const int32_t* starts, const grkv_chunk* chunk, void* o, float* lse,
                         void* stream, void* workspace, size_t workspace_bytes);

size_t grkv_chunk_attention_workspace_bytes(const grkv_pages* pages, const grkv_step* step,
                                            const grkv_chunk* chunk);

/* These are asynchronous on stream, allocate nothing and may be captured.  Errors: those of the
 * calls on pages; GRKV_ERR_INVALID for null pointers and sizes out of range (sequences *
 * heads >= 2^24, tokens * heads or tokens * head_dim >= 2^31, heads of a rotation,
 * or 2 heads + q_heads of a store, > 65535, tokens * heads * group >= 2^30, a chunk call of 2^24
 * row tiles or more); GRKV_ERR_UNSUPPORTED for head_dim > 32768 of grkv_rotary.  A rotation's scale
 * and frequencies are taken as they are. */

/* Workspace bytes grkv_compress needs for this shape; 0 if the shape is
 * invalid or unsupported. */
size_t grkv_workspace_bytes(const grkv_problem* prob, int64_t n,
                            int32_t window, int32_t budget);

/* Byte offsets, inside the workspace, of intermediates that remain readable
 * after grkv_compress returns (mp = m rounded up to 32, 64, 128 or 256; rows
 * m..mp-1 are padding; P = n - w):
 *   lse      double [U][mp]     natural log-sum-exp of each window row over the
 *                               full cache (window attention normaliser)
 *   y        float  [U][mp][d]  Y = A V, the full-cache window attention output
 *   score    float  [U][P]      SnapKV score s_j = sum_r A[r][j]
 *   pooled   float  [U][P]      pooled score p_j
 *   fixed    uint8  [U][c]      1 where the retained slot is fixed
 *   resid    float  [U][mp][d]  R = Y - X V0
 *   gram     float  [U][mp][mp] N = X_G X_G^T + lambda I (padding rows: identity)
 *   z        float  [U][d][mp]  Z^T, Z = N^-1 R
 * Returns GRKV_OK, or GRKV_ERR_INVALID / GRKV_ERR_UNSUPPORTED like
 * grkv_compress. */
typedef struct {
  size_t lse, y, score, pooled, fixed, resid, gram, z;
  size_t total;
} grkv_layout;

int grkv_workspace_layout(const grkv_problem* prob, int64_t n, int32_t window,
                          int32_t budget, grkv_layout* layout);

/* The default options (see grkv_options). */
void grkv_default_options(grkv_options* opt);

/* Static description of a return code; never NULL. */
const char* grkv_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* GRKV_H */
