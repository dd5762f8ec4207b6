// C entry points of the pages of a cache and of the attention that reads them:
// argument checks on the host, then the launches.
#include "grkv_internal.h"

using namespace grkv;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

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
  PagesCall c = {};
  c.op = kPagesFree;
  c.pages = pages;
  c.entries = entries;
  return run(c, stream);
}

}  // extern "C"
