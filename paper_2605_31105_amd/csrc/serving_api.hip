// C entry points of the pages of a cache and of the attention that reads them:
// argument checks on the host, then the launches.
#include <math.h>

#include "grkv_internal.h"

using namespace grkv;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Blocks of 256 threads in a launch, which has fewer than 2^32 threads.
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;

// Heads of a launch of rotated rows (its grid's second size).
constexpr int64_t kMostHeads = 65535;

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

int check_step(const grkv_pages* pg, const grkv_step* st) {
  const int ok = check_pages(pg);
  if (ok != GRKV_OK) return ok;
  if (!st || st->sequences < 0 || st->heads < 1 || st->tokens < 0) return GRKV_ERR_INVALID;
  if (st->units && st->unit_stride < st->heads) return GRKV_ERR_INVALID;
  // (both limits: launches, and the sums of pages in extend.hip)
  if ((int64_t)st->sequences * st->heads > kMostBlocks) return GRKV_ERR_INVALID;
  return (int64_t)st->tokens * st->heads >= (int64_t(1) << 31) ? GRKV_ERR_INVALID : GRKV_OK;
}

struct ChunkCall {
  AttendK a;
  ChunkPlan plan;
};

int make_chunk(const grkv_pages* pg, const grkv_step* st, const grkv_chunk* ch, ChunkCall* c) {
  const int ok = check_step(pg, st);
  if (ok != GRKV_OK) return ok;
  if (!ch || ch->group < 1 || ch->longest < 1 || ch->window < 0 || ch->n_sink < 0) return GRKV_ERR_INVALID;
  const int64_t per = (int64_t)st->heads * ch->group;
  if (per >= (int64_t(1) << 30) || per * st->tokens >= (int64_t(1) << 30)) return GRKV_ERR_INVALID;
  const int64_t cap = (int64_t)pg->max_pages * pg->page_size;
  const int window = window_of(ch->window, cap);
  // (a job's rows, 128 at most, lie at 128 / group + 2 positions or fewer)
  const int64_t near = (int64_t)ch->n_sink + window + 128 / ch->group + 2;
  c->plan = chunk_plan(st, ch, pg->head_dim, pg->dtype, window > 0 && near < cap ? near : cap);
  if (c->plan.jobs > kMostBlocks) return GRKV_ERR_INVALID;
  AttendK& a = c->a;
  a = AttendK{};
  a.k = pg->k;
  a.v = pg->v;
  a.group = ch->group;
  a.window = window;
  a.n_sink = sinks_of(ch->n_sink);
  a.table = pg->table;
  a.lens = pg->lens;
  a.units = st->units;
  a.max_pages = pg->max_pages;
  a.shift = __builtin_ctz((unsigned)pg->page_size);
  a.pages = pg->pages;
  a.pool_units = pg->units;
  a.unit_stride = st->unit_stride;
  a.sequences = st->sequences;
  a.heads = st->heads;
  a.q_heads = st->heads * ch->group;
  a.longest = ch->longest;
  a.step_tokens = st->tokens;
  return GRKV_OK;
}

// A rotation of rows of d columns.
int check_rotation(const grkv_rotation* rot, const int32_t* positions, int32_t d) {
  if (!rot || !rot->freqs || !positions || !aligned(rot->freqs, 8)) return GRKV_ERR_INVALID;
  if (rot->dims < 2 || rot->dims > d || rot->dims % 2 != 0) return GRKV_ERR_INVALID;
  return GRKV_OK;
}

bool rows_ok(const grkv_rows* r, int dtype) {
  return r && r->data && aligned(r->data, dtype == GRKV_BF16 ? 2 : 4);
}

RotaryK rotary_of(const grkv_rows* x, const grkv_rows* y, int32_t tokens, int32_t heads, int32_t d,
                  const int32_t* positions, const grkv_rotation* rot) {
  RotaryK r = {};
  if (x) r.x = *x;
  if (y) r.y = *y;
  r.tokens = (uint32_t)tokens;
  r.heads = heads;
  r.d = d;
  if (rot) {
    r.dims = rot->dims;
    r.interleaved = rot->interleaved != 0;
    r.inverse = rot->inverse != 0;
    r.scale = rot->scale;
    r.freqs = rot->freqs;
    r.positions = positions;
  }
  return r;
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

size_t grkv_pages_extend_workspace_bytes(const grkv_pages* pages, const grkv_step* step) {
  if (check_step(pages, step) != GRKV_OK) return 0;
  return extend_layout(pages, step->sequences, step->heads).total;
}

int grkv_pages_extend(const grkv_pages* pages, const grkv_step* step, const int32_t* counts,
                      const int32_t* seen, int32_t* starts, int32_t* positions, int64_t* slots,
                      int32_t* status, void* stream, void* workspace, size_t workspace_bytes) {
  const int st = check_step(pages, step);
  if (st != GRKV_OK) return st;
  if (step->sequences == 0) return GRKV_OK;
  if (!counts || !starts || (step->tokens > 0 && (!positions || !slots))) return GRKV_ERR_INVALID;
  if (!workspace || !aligned(workspace, 256)) return GRKV_ERR_INVALID;
  if (workspace_bytes < grkv_pages_extend_workspace_bytes(pages, step)) return GRKV_ERR_WORKSPACE;
  return launch_extend(pages, step, counts, seen, starts, positions, slots, status, workspace,
                       (hipStream_t)stream) == hipSuccess ? GRKV_OK : GRKV_ERR_HIP;
}

int grkv_rotary(const grkv_rows* x, const grkv_rows* y, int32_t tokens, int32_t heads,
                int32_t head_dim, int32_t dtype, const int32_t* positions,
                const grkv_rotation* rotation, void* stream) {
  if (tokens < 0 || heads < 0 || heads > kMostHeads || head_dim < 2) return GRKV_ERR_INVALID;
  if (dtype != GRKV_BF16 && dtype != GRKV_F32) return GRKV_ERR_INVALID;
  if (head_dim > 32768) return GRKV_ERR_UNSUPPORTED;
  if ((int64_t)tokens * head_dim >= (int64_t(1) << 31)) return GRKV_ERR_INVALID;
  if (tokens == 0 || heads == 0) return GRKV_OK;
  const int st = check_rotation(rotation, positions, head_dim);
  if (st != GRKV_OK) return st;
  if (!rows_ok(x, dtype) || !rows_ok(y, dtype)) return GRKV_ERR_INVALID;
  return launch_rotary(rotary_of(x, y, tokens, heads, head_dim, positions, rotation), dtype,
                       (hipStream_t)stream) == hipSuccess ? GRKV_OK : GRKV_ERR_HIP;
}

int grkv_rotary_freqs(int32_t dims, double base, int32_t method, double factor, double length,
                      double low, double high, double* freqs) {
  if (dims < 2 || dims % 2 != 0 || dims > 32768 || !freqs || !(base > 0.0) || !isfinite(base)) return GRKV_ERR_INVALID;
  if (method < GRKV_ROTARY_PLAIN || method > GRKV_ROTARY_PARTS) return GRKV_ERR_INVALID;
  if (method != GRKV_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return GRKV_ERR_INVALID;
  if (method == GRKV_ROTARY_PARTS &&
      (!(length > 0.0) || !isfinite(length) || !(low >= 0.0) || !(high > low) || !isfinite(high)))
    return GRKV_ERR_INVALID;
  if (method == GRKV_ROTARY_BASE && dims > 2) base *= pow(factor, (double)dims / (dims - 2));
  if (!isfinite(base)) return GRKV_ERR_INVALID;
  for (int i = 0; i < dims / 2; ++i) {
    double f = pow(base, -2.0 * i / dims);
    if (method == GRKV_ROTARY_LINEAR) f /= factor;
    if (method == GRKV_ROTARY_PARTS) {
      const double turns = length * f / 6.283185307179586477;
      double stay = (turns - low) / (high - low);
      stay = stay < 0.0 ? 0.0 : stay > 1.0 ? 1.0 : stay;
      f = f * stay + f / factor * (1.0 - stay);
    }
    // (constants far apart: a frequency of 0 would leave its pair without a position)
    if (!(f > 0.0) || !isfinite(f)) return GRKV_ERR_INVALID;
    freqs[i] = f;
  }
  return GRKV_OK;
}

int grkv_pages_store(const grkv_pages* pages, int32_t tokens, int32_t heads, const int64_t* slots,
                     int64_t slot_stride, const grkv_rows* k, const grkv_rows* v, int32_t dtype,
                     const grkv_rows* q, const grkv_rows* q_out, int32_t q_heads,
                     const int32_t* positions, const grkv_rotation* rotation, void* stream) {
  int st = check_pages(pages);
  if (st != GRKV_OK) return st;
  if (tokens < 0 || heads < 0 || q_heads < 0 || slot_stride < heads) return GRKV_ERR_INVALID;
  if (2 * (int64_t)heads + q_heads > kMostHeads) return GRKV_ERR_INVALID;
  if (dtype != GRKV_BF16 && dtype != GRKV_F32) return GRKV_ERR_INVALID;
  if ((int64_t)tokens * pages->head_dim >= (int64_t(1) << 31)) return GRKV_ERR_INVALID;
  if (!rotation) q_heads = 0;
  if (tokens == 0 || heads + q_heads == 0) return GRKV_OK;
  if (rotation && (st = check_rotation(rotation, positions, pages->head_dim)) != GRKV_OK) return st;
  if (heads > 0 && (!slots || !rows_ok(k, dtype) || !rows_ok(v, dtype))) return GRKV_ERR_INVALID;
  if (q_heads > 0 && (!rows_ok(q, dtype) || !rows_ok(q_out, dtype))) return GRKV_ERR_INVALID;
  StoreK a = {};
  a.r = rotary_of(q_heads > 0 ? q : nullptr, q_heads > 0 ? q_out : nullptr, tokens, q_heads, pages->head_dim,
                  positions, rotation);
  if (heads > 0) {
    a.k = *k;
    a.v = *v;
  }
  a.pool_k = pages->k;
  a.pool_v = pages->v;
  a.heads = heads;
  a.slots = slots;
  a.slot_stride = slot_stride;
  a.rows = (int64_t)pages->pages * pages->page_size;
  return launch_store(a, dtype, pages->dtype, (hipStream_t)stream) == hipSuccess ? GRKV_OK : GRKV_ERR_HIP;
}

size_t grkv_chunk_attention_workspace_bytes(const grkv_pages* pages, const grkv_step* step,
                                            const grkv_chunk* chunk) {
  ChunkCall c;
  if (make_chunk(pages, step, chunk, &c) != GRKV_OK) return 0;
  return c.plan.total;
}

int grkv_chunk_attention(const void* q, const grkv_pages* pages, const grkv_step* step,
                         const int32_t* starts, const grkv_chunk* chunk, void* o, float* lse,
                         void* stream, void* workspace, size_t workspace_bytes) {
  ChunkCall c;
  const int st = make_chunk(pages, step, chunk, &c);
  if (st != GRKV_OK) return st;
  if (step->sequences == 0 || step->tokens == 0) return GRKV_OK;
  if (!q || !o || !starts || !aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4)) return GRKV_ERR_INVALID;
  if (!workspace || !aligned(workspace, 256)) return GRKV_ERR_INVALID;
  if (workspace_bytes < c.plan.total) return GRKV_ERR_WORKSPACE;
  c.a.q = q;
  c.a.o = o;
  c.a.lse = lse;
  c.a.starts = starts;
  return launch_chunk(c.a, c.plan, pages->head_dim, pages->dtype, workspace, (hipStream_t)stream) == hipSuccess
             ? GRKV_OK : GRKV_ERR_HIP;
}

}  // extern "C"
