// C entry points of the pages of a cache and of the attention that reads them:
// argument checks on the host, then the launches.
#include "grkv_internal.h"

using namespace grkv;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Blocks of 256 threads in a launch, which has fewer than 2^32 threads.
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;

// Rows and elements of q within the kernels' indices.
bool sizes_ok(int64_t entries, int64_t group, int64_t tokens, int64_t d) {
  return group * tokens < (int64_t(1) << 30) &&
         (entries == 0 || group * tokens * d < (int64_t(1) << 40) / entries);
}

int check_pages(const grkv_pages* pg) {
  if (!pg || !pg->k || !pg->v || !pg->table || !pg->lens || !pg->refs || !pg->free_bits)
    return GRKV_ERR_INVALID;
  if (!aligned(pg->k, 16) || !aligned(pg->v, 16)) return GRKV_ERR_INVALID;
  if (pg->pages < 1 || pg->pages > (1 << 30) || pg->units < 1 || pg->max_pages < 1)
    return GRKV_ERR_INVALID;
  if (pg->dtype != GRKV_BF16 && pg->dtype != GRKV_F32) return GRKV_ERR_INVALID;
  if (pg->page_size < 16 || pg->page_size > 1024 || (pg->page_size & (pg->page_size - 1)) != 0)
    return GRKV_ERR_UNSUPPORTED;
  if (pg->head_dim != 64 && pg->head_dim != 128) return GRKV_ERR_UNSUPPORTED;
  if ((int64_t)pg->max_pages * pg->page_size > (int64_t(1) << 30)) return GRKV_ERR_INVALID;
  return GRKV_OK;
}

int check_entries(const grkv_pages* pg, const grkv_page_entries* en, bool rows) {
  const int st = check_pages(pg);
  if (st != GRKV_OK) return st;
  if (!en || en->entries < 0) return GRKV_ERR_INVALID;
  if (!rows) return GRKV_OK;
  if (en->rows < 0 || en->source_rows < 0) return GRKV_ERR_INVALID;
  if ((int64_t)en->entries * ((int64_t)en->rows + pg->page_size) >= (int64_t(1) << 31))
    return GRKV_ERR_INVALID;
  return GRKV_OK;
}

int check_workspace(const grkv_pages* pg, const grkv_page_entries* en, const void* ws, size_t bytes) {
  if (en->entries == 0) return GRKV_OK;
  if (!ws || !aligned(ws, 256)) return GRKV_ERR_INVALID;
  return bytes < grkv_pages_workspace_bytes(pg, en->entries) ? GRKV_ERR_WORKSPACE : GRKV_OK;
}

int run(const PagesCall& c, void* stream) {
  return launch_pages(c, (hipStream_t)stream) == hipSuccess ? GRKV_OK : GRKV_ERR_HIP;
}

// The window as the kernels take it: one that holds every slot is none.  (A window
// below 2^30 also keeps differences of positions within 32 bits.)
int window_of(int window, int64_t slots) { return window < slots ? window : 0; }
int sinks_of(int n_sink) { return n_sink < (1 << 30) ? n_sink : 1 << 30; }

// A call's sizes and plan.  A call without splits still asks for 256 bytes, so
// that 0 says "invalid".
struct TreeCall {
  AttendK a;
  AttendPlan plan;
};

int make_tree(const grkv_pages* pg, const grkv_tree* tr, TreeCall* c) {
  const int st = check_pages(pg);
  if (st != GRKV_OK) return st;
  if (!tr || tr->entries < 0 || tr->group < 1 || tr->tokens < 1 || tr->window < 0 || tr->n_sink < 0)
    return GRKV_ERR_INVALID;
  if (tr->tokens > 64) return GRKV_ERR_UNSUPPORTED;
  if (tr->parents && tr->entries > 0 && (tr->trees < 1 || tr->entries % tr->trees != 0))
    return GRKV_ERR_INVALID;
  if (!sizes_ok(tr->entries, tr->group, tr->tokens, pg->head_dim)) return GRKV_ERR_INVALID;
  const int64_t cap = (int64_t)pg->max_pages * pg->page_size;
  const int window = window_of(tr->window, cap);
  const int64_t near = (int64_t)tr->n_sink + window + tr->tokens;
  c->plan = attend_plan(tr->entries > 0 ? tr->entries : 1, tr->group, tr->tokens, pg->head_dim,
                        pg->dtype, window > 0 && near < cap ? near : cap, window == 0);
  if (c->plan.blocks > kMostBlocks) return GRKV_ERR_INVALID;
  AttendK& a = c->a;
  a = AttendK{};
  a.k = pg->k;
  a.v = pg->v;
  a.entries = tr->entries;
  a.group = tr->group;
  a.tokens = tr->tokens;
  a.window = window;
  a.n_sink = sinks_of(tr->n_sink);
  a.table = pg->table;
  a.lens = pg->lens;
  a.units = tr->units;
  a.counts = tr->counts;
  a.parents = tr->parents;
  a.per_tree = tr->parents && tr->entries > 0 ? tr->entries / tr->trees : 1;
  a.max_pages = pg->max_pages;
  a.shift = __builtin_ctz((unsigned)pg->page_size);
  a.pages = pg->pages;
  a.pool_units = pg->units;
  return GRKV_OK;
}

int make_sink(const grkv_problem* prob, int64_t n, int32_t nq, int32_t window, int32_t n_sink,
              TreeCall* c) {
  if (!prob || prob->units < 1 || prob->group < 1) return GRKV_ERR_INVALID;
  if (prob->dtype != GRKV_BF16 && prob->dtype != GRKV_F32) return GRKV_ERR_INVALID;
  if (nq < 1 || nq > n || n > (int64_t(1) << 30) || window < 0 || n_sink < 0) return GRKV_ERR_INVALID;
  if (prob->head_dim != 64 && prob->head_dim != 128) return GRKV_ERR_UNSUPPORTED;
  if (!sizes_ok(prob->units, prob->group, nq, prob->head_dim)) return GRKV_ERR_INVALID;
  window = window_of(window, n);
  // (a block's rows, 128 at most, lie at 128 / group + 2 positions or fewer)
  const int64_t near = (int64_t)n_sink + window + (nq < 128 / prob->group + 2 ? nq : 128 / prob->group + 2);
  c->plan = attend_plan(prob->units, prob->group, nq, prob->head_dim, prob->dtype,
                        window > 0 && near < n ? near : n, false);
  if (c->plan.blocks > kMostBlocks) return GRKV_ERR_INVALID;
  AttendK& a = c->a;
  a = AttendK{};
  a.entries = prob->units;
  a.group = prob->group;
  a.tokens = nq;
  a.window = window;
  a.n_sink = sinks_of(n_sink);
  a.n = (int)n;
  return GRKV_OK;
}

size_t workspace_of(const AttendPlan& p) { return p.total > 256 ? p.total : 256; }

int run_attend(const TreeCall& c, int d, int dtype, void* stream, void* ws, size_t bytes) {
  if (!ws || !aligned(ws, 256)) return GRKV_ERR_INVALID;
  if (bytes < workspace_of(c.plan)) return GRKV_ERR_WORKSPACE;
  return launch_attend(c.a, c.plan, d, dtype, ws, (hipStream_t)stream) == hipSuccess ? GRKV_OK
                                                                                     : GRKV_ERR_HIP;
}

}  // namespace

extern "C" {

size_t grkv_pages_workspace_bytes(const grkv_pages* pages, int32_t entries) {
  if (check_pages(pages) != GRKV_OK || entries < 0) return 0;
  return pages_layout(pages, entries).total;
}

int grkv_pages_init(const grkv_pages* pages, void* stream) {
  const int st = check_pages(pages);
  if (st != GRKV_OK) return st;
  PagesCall c = {};
  c.op = kPagesInit;
  c.pages = pages;
  return run(c, stream);
}

int grkv_pages_append(const grkv_pages* pages, const grkv_page_entries* entries, const void* k,
                      int32_t k_dtype, const void* v, int32_t v_dtype, void* stream,
                      void* workspace, size_t workspace_bytes) {
  int st = check_entries(pages, entries, true);
  if (st != GRKV_OK) return st;
  if (entries->entries > 0 && entries->rows > 0 && entries->source_rows > 0 &&
      (!k || !v || !aligned(k, 16) || !aligned(v, 16)))
    return GRKV_ERR_INVALID;
  if ((k_dtype != GRKV_BF16 && k_dtype != GRKV_F32) || (v_dtype != GRKV_BF16 && v_dtype != GRKV_F32))
    return GRKV_ERR_INVALID;
  st = check_workspace(pages, entries, workspace, workspace_bytes);
  if (st != GRKV_OK) return st;
  PagesCall c = {};
  c.op = kPagesAppend;
  c.pages = pages;
  c.entries = entries;
  c.k = k;
  c.v = v;
  c.k_dtype = k_dtype;
  c.v_dtype = v_dtype;
  c.workspace = workspace;
  return run(c, stream);
}

int grkv_pages_fork(const grkv_pages* pages, const grkv_page_entries* entries, const int32_t* dst,
                    void* stream, void* workspace, size_t workspace_bytes) {
  int st = check_entries(pages, entries, false);
  if (st != GRKV_OK) return st;
  if ((int64_t)entries->entries * pages->page_size >= (int64_t(1) << 31)) return GRKV_ERR_INVALID;
  if (entries->entries > kMostBlocks) return GRKV_ERR_INVALID;
  if (entries->entries > 0 && !dst) return GRKV_ERR_INVALID;
  st = check_workspace(pages, entries, workspace, workspace_bytes);
  if (st != GRKV_OK) return st;
  PagesCall c = {};
  c.op = kPagesFork;
  c.pages = pages;
  c.entries = entries;
  c.dst = dst;
  c.workspace = workspace;
  return run(c, stream);
}

int grkv_pages_compact(const grkv_pages* pages, const grkv_page_entries* entries,
                       const int32_t* dst, const int32_t* keep, const int32_t* idx, void* stream,
                       void* workspace, size_t workspace_bytes) {
  int st = check_entries(pages, entries, true);
  if (st != GRKV_OK) return st;
  if (entries->entries > kMostBlocks) return GRKV_ERR_INVALID;
  if (entries->entries > 0 && entries->rows > 0 && entries->source_rows > 0 && !idx)
    return GRKV_ERR_INVALID;
  st = check_workspace(pages, entries, workspace, workspace_bytes);
  if (st != GRKV_OK) return st;
  PagesCall c = {};
  c.op = kPagesCompact;
  c.pages = pages;
  c.entries = entries;
  c.dst = dst;
  c.keep = keep;
  c.idx = idx;
  c.workspace = workspace;
  return run(c, stream);
}

int grkv_pages_free(const grkv_pages* pages, const grkv_page_entries* entries, void* stream) {
  const int st = check_entries(pages, entries, false);
  if (st != GRKV_OK) return st;
  if (entries->entries > kMostBlocks) return GRKV_ERR_INVALID;
  PagesCall c = {};
  c.op = kPagesFree;
  c.pages = pages;
  c.entries = entries;
  return run(c, stream);
}

size_t grkv_tree_attention_workspace_bytes(const grkv_pages* pages, const grkv_tree* tree) {
  TreeCall c;
  if (make_tree(pages, tree, &c) != GRKV_OK) return 0;
  return workspace_of(c.plan);
}

int grkv_tree_attention(const void* q, const grkv_pages* pages, const grkv_tree* tree, void* o,
                        float* lse, void* stream, void* workspace, size_t workspace_bytes) {
  TreeCall c;
  const int st = make_tree(pages, tree, &c);
  if (st != GRKV_OK) return st;
  if (tree->entries == 0) return GRKV_OK;
  if (!q || !o || !aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4)) return GRKV_ERR_INVALID;
  c.a.q = q;
  c.a.o = o;
  c.a.lse = lse;
  return run_attend(c, pages->head_dim, pages->dtype, stream, workspace, workspace_bytes);
}

size_t grkv_sink_attention_workspace_bytes(const grkv_problem* prob, int64_t n, int32_t nq,
                                           int32_t window, int32_t n_sink) {
  TreeCall c;
  if (make_sink(prob, n, nq, window, n_sink, &c) != GRKV_OK) return 0;
  return workspace_of(c.plan);
}

int grkv_sink_attention(const void* q, const void* K, const void* V, int64_t n, int32_t nq,
                        int32_t window, int32_t n_sink, void* stream, const grkv_problem* prob,
                        void* o, float* lse, void* workspace, size_t workspace_bytes) {
  TreeCall c;
  const int st = make_sink(prob, n, nq, window, n_sink, &c);
  if (st != GRKV_OK) return st;
  if (!q || !K || !V || !o) return GRKV_ERR_INVALID;
  if (!aligned(q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(o, 16) || !aligned(lse, 4))
    return GRKV_ERR_INVALID;
  c.a.q = q;
  c.a.k = K;
  c.a.v = V;
  c.a.o = o;
  c.a.lse = lse;
  return run_attend(c, prob->head_dim, prob->dtype, stream, workspace, workspace_bytes);
}

}  // extern "C"
