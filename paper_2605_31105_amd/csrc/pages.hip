// Pages of a cache: rows stored in, branched over, picked from and released
// from the pages of one pool (grkv_pages_append, _fork, _compact, _free).
//
// A call that needs new pages is a plan and a copy:
//  * plan_kernel, one block: checks every entry, counts the pages it needs
//    (a block scan in the order of the entries), takes the free pages of lowest
//    number from the bitmap (a block scan over the words' bit counts), and
//    writes one job per entry.  One block, because the pages that an entry
//    gets depend on all entries before it; a scan over bits, because a stack
//    of free pages would hold them in the order in which atomics arrived, so
//    two runs of the same calls would differ.
//  * append_kernel / move_kernel: the rows, 16 bytes of K and of V per thread
//    and step; which entry, row and page a thread serves follows from its
//    index and the entry's job.  What bounds them is HBM (each row read and
//    written once) or, for the few rows of a decoding step, the launches.
//  * commit_kernel (fork, compact): the table rows and reference counts, after
//    the rows that move_kernel reads through the old table are copied.
#include "grkv_device.h"
#include "grkv_internal.h"

namespace grkv {
namespace {

constexpr int kPlanTh = 1024;
constexpr int kCopyTh = 256;
constexpr int kNoOwner = 0x7fffffff;
constexpr int kOwnerUnits = 8192;   // units of a pool whose owners fit the plan's LDS

// What an entry of a call does, written by the plan.  n1 < 0: nothing (a
// refused entry).
struct PageJob {
  int32_t src, dst;
  int32_t n0, n1;      // rows of src before, rows of dst after
  int32_t keep;        // rows of dst that are the same slots of src (append: n0)
  int32_t first;       // first page of dst that is new
  int32_t last;        // pages of dst after
  int32_t off;         // the new pages are ids[off ..]
  int64_t start;       // first row (index) in the packed source
};

struct PagesK {
  grkv_pages pg;
  int shift;            // log2 page_size
  PagesOp op;
  int entries, rows;
  const int32_t* units;
  const int32_t* dst;
  const int32_t* counts;
  const int32_t* keep;
  const int64_t* starts;
  int64_t source_rows;
  int32_t* status;
  int32_t* owner;       // [units] lowest entry that writes the unit
  PageJob* jobs;        // [entries]
  int32_t* ids;         // [pages] pages handed out, in order
};

__device__ __forceinline__ int load_agent(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive scan over the block of the plan.  Calls in a row take the halves of
// `scratch` in turn (`turn` 0, 1, 0, ..), so one barrier each is enough.
template <typename T>
__device__ __forceinline__ T plan_scan(T v, T (*scratch)[kPlanTh / 64], int turn, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T incl = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T t = __shfl_up(incl, off);
    if (lane >= off) incl += t;
  }
  if (lane == 63) scratch[turn & 1][wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kPlanTh / 64; ++k) {
    const T s = scratch[turn & 1][k];
    if (k < wave) before += s;
    all += s;
  }
  *total = all;
  return before + incl - v;
}

// The plan of a call, by one block.  Most calls have at most one entry per thread;
// then a job stays in its thread's registers until it is complete.
__device__ __forceinline__ void make_plan_block(const PagesK& a) {
  __shared__ int owner_s[kOwnerUnits];
  // (an entry may ask for 2^26 pages: their sums take 64 bits)
  __shared__ unsigned long long scratch[2][kPlanTh / 64];
  __shared__ uint32_t scratch32[2][kPlanTh / 64];
  __shared__ uint32_t taken_s[kPlanTh], rank_s[kPlanTh];   // pages taken of a word, the first one's rank
  __shared__ int used_s;
  const int tid = threadIdx.x, lane = tid & 63;
  const int ps = 1 << a.shift;
  const int64_t cap = (int64_t)a.pg.max_pages << a.shift;
  auto unit_of = [&](int i) { return a.units ? a.units[i] : i; };
  auto in_pool = [&](int u) { return (unsigned)u < (unsigned)a.pg.units; };

  // (read here, while the entries are)
  const int words = (a.pg.pages + 31) / 32;
  const uint32_t bits0 = tid < words ? a.pg.free_bits[tid] : 0u;

  // owner of a unit: the lowest entry that writes it (in LDS where the pool is
  // small; entry i is unit i's without lists of units)
  const bool listed = a.units || a.dst, small = a.pg.units <= kOwnerUnits;
  if (tid == 0) used_s = 0;
  if (listed && small) {
    for (int u = tid; u < a.pg.units; u += kPlanTh) owner_s[u] = kNoOwner;
    __syncthreads();
    for (int i = tid; i < a.entries; i += kPlanTh) {
      const int w = a.dst ? a.dst[i] : unit_of(i);
      if (in_pool(w)) atomicMin(owner_s + w, i);
    }
  } else if (listed) {
    for (int i = tid; i < a.entries; i += kPlanTh) {
      const int u = unit_of(i), w = a.dst ? a.dst[i] : u;
      if (in_pool(u)) a.owner[u] = kNoOwner;
      if (in_pool(w)) a.owner[w] = kNoOwner;
    }
    __syncthreads();
    for (int i = tid; i < a.entries; i += kPlanTh) {
      const int w = a.dst ? a.dst[i] : unit_of(i);
      if (in_pool(w)) atomicMin(a.owner + w, i);
    }
  }
  __syncthreads();
  auto owner = [&](int u) { return small ? owner_s[u] : load_agent(a.owner + u); };

  // each entry's status and job, but for the pages it gets
  PageJob j;
  int st = GRKV_PAGES_OK;
  unsigned long long need_all = 0;
  int turn = 0;
  for (int i0 = 0; i0 < a.entries; i0 += kPlanTh) {
    const int i = i0 + tid;
    st = GRKV_PAGES_OK;
    j = PageJob{};
    if (i < a.entries) {
      j.src = unit_of(i);
      j.dst = a.dst ? a.dst[i] : j.src;
      const bool moved = j.dst != j.src;
      if (!in_pool(j.src) || !in_pool(j.dst) ||
          (listed && (owner(j.dst) != i || (moved && owner(j.src) != kNoOwner)))) {
        st = GRKV_PAGES_UNIT;
      } else {
        j.n0 = a.pg.lens[j.src];
        const int there = moved ? a.pg.lens[j.dst] : 0;
        int count = a.op == kPagesFork ? 0 : a.rows;
        if (a.counts) count = min(max(a.counts[i], 0), a.rows);
        j.start = a.starts ? a.starts[i] : (int64_t)i * a.rows;
        j.keep = a.op != kPagesCompact ? j.n0 : a.keep ? a.keep[i] : 0;
        const int64_t n1 = (int64_t)j.keep + count;
        if (j.n0 < 0 || j.n0 > cap || there != 0) {
          st = GRKV_PAGES_UNIT;
        } else if (j.keep < 0 || j.keep > j.n0 ||
                   (count > 0 && (j.start < 0 || j.start > a.source_rows - count))) {
          st = GRKV_PAGES_RANGE;
        } else if (n1 > cap) {
          st = GRKV_PAGES_LENGTH;
        } else {
          j.n1 = (int)n1;
          j.last = (int)((n1 + ps - 1) >> a.shift);
          if (a.op == kPagesAppend) {
            j.first = (j.n0 + ps - 1) >> a.shift;
          } else {
            j.first = j.keep >> a.shift;
            // slots taken back in place: a last page of the unit's own stays
            if (!moved && count == 0 && (j.keep & (ps - 1)) != 0) {
              const int p = a.pg.table[(size_t)j.src * a.pg.max_pages + j.first];
              if ((unsigned)p < (unsigned)a.pg.pages && a.pg.refs[p] == 1) ++j.first;
            }
          }
        }
      }
      if (st != GRKV_PAGES_OK) j.n1 = -1;
    }
    const unsigned long long need = st == GRKV_PAGES_OK ? max(j.last - j.first, 0) : 0;
    unsigned long long total;
    const unsigned long long off = need_all + plan_scan(need, scratch, turn++, &total);
    need_all += total;
    // (an entry whose pages end past the pool's last is refused below)
    j.off = (int)(off < (unsigned)a.pg.pages ? off : (unsigned)a.pg.pages);
    if (a.entries > kPlanTh && i < a.entries) {
      a.jobs[i] = j;
      if (a.status) a.status[i] = st;
    }
  }

  // the lowest free pages, as many as are asked for.  A thread takes a word of 32
  // pages; the numbers are written two words at a time by a wave, neighbouring lanes
  // neighbouring numbers, the waves in turn (plans of 2048 and 34k pages 6.3 and 12.4 us;
  // each wave the words that its lanes hold, 10.1 and 19.2)
  const uint32_t want = (uint32_t)(need_all < (unsigned)a.pg.pages ? need_all : (unsigned)a.pg.pages);
  uint32_t found = 0;
  for (int w0 = 0; w0 < words && found < want; w0 += kPlanTh) {
    const int w = w0 + tid;
    const uint32_t bits = w0 == 0 ? bits0 : w < words ? a.pg.free_bits[w] : 0u;
    uint32_t total;
    const uint32_t r0 = found + plan_scan((uint32_t)__popc(bits), scratch32, turn++, &total);
    uint32_t left = 0;
    if (r0 + __popc(bits) > want) {   // the last word taken from, and those behind it
      left = bits;
      for (uint32_t r = r0; r < want; ++r) left &= left - 1;
    }
    if (left != bits) a.pg.free_bits[w] = left;
    taken_s[tid] = bits ^ left;
    rank_s[tid] = r0;
    __syncthreads();   // (read before the next scan's barrier)
    const int here = min(words - w0, kPlanTh), bit = lane & 31;
    for (int k = (tid >> 6) * 2 + (lane >> 5); k < here; k += kPlanTh / 32) {
      const uint32_t t = taken_s[k];
      if (t >> bit & 1) a.ids[rank_s[k] + __popc(t & ((1u << bit) - 1))] = 32 * (w0 + k) + bit;
    }
    found += total;
  }
  found = found < want ? found : want;

  // entries past the free pages are refused; lengths
  int used = 0;
  for (int i = tid; i < a.entries; i += kPlanTh) {
    if (a.entries > kPlanTh) {
      j = a.jobs[i];
      st = GRKV_PAGES_OK;   // (a refused entry's status is written)
    }
    const int need = j.n1 < 0 ? 0 : j.last - j.first;
    if (need > 0) {
      if ((uint64_t)j.off + need > found) {
        j.n1 = -1;
        st = GRKV_PAGES_FULL;
      } else {
        used = max(used, j.off + need);
      }
    }
    if (j.n1 >= 0) a.pg.lens[j.dst] = j.n1;
    if (a.entries <= kPlanTh || st != GRKV_PAGES_OK) {
      a.jobs[i] = j;
      if (a.status) a.status[i] = st;
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) used = max(used, __shfl_xor(used, k));
  if (lane == 0 && used > 0) atomicMax(&used_s, used);
  __syncthreads();
  // pages taken for refused entries go back
  for (uint32_t r = used_s + tid; r < found; r += kPlanTh)
    atomicOr(a.pg.free_bits + (a.ids[r] >> 5), 1u << (a.ids[r] & 31));
}

__global__ __launch_bounds__(kPlanTh) void plan_kernel(PagesK a) { make_plan_block(a); }

// The rows of a launch: row g is row (g % tile + tile * ((g / tile) % per)) of
// entry g / tile / per, so that the rows of one tile are neighbours and a
// block serves many entries where each has few.  tile is a power of two.
struct RowMap {
  int tile_shift;
  uint32_t per;       // tiles of an entry
  uint32_t rows;      // rows of the launch, padded: entries * per << tile_shift
};

__device__ __forceinline__ void map_row(const RowMap& m, uint32_t g, int* entry, int* row) {
  const uint32_t t = g >> m.tile_shift, e = t / m.per;
  *entry = (int)e;
  *row = (int)(((t - e * m.per) << m.tile_shift) | (g & ((1u << m.tile_shift) - 1)));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Source values as 16 bytes of the pool's type (rounded to nearest even), so that the
// stores of a wave are whole lines (32 bytes per thread, in two stores of every other 16:
// 2 units' 103k rows of float32 in 190 us).
// LONG: of a long call, whose rows pass the caches on their way out (over pools used
// in turn, a layer's 32k rows stored, thinned and released 80 -> 78 us, ragged results
// 113 -> 110; read so too, 76 and 111); moved rows always do (8 units of 16k rows thinned
// to 12k 72.6 -> 69.0, 500 of 300 to 500 rows to 150 68 -> 62).
template <bool LONG>
__device__ __forceinline__ void store16(void* p, u32x4 v) {
  if constexpr (LONG) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

template <bool LONG, typename S, typename T>
__device__ __forceinline__ void copy16(const S* src, T* dst) {
  if constexpr (sizeof(S) == sizeof(T)) {
    store16<LONG>(dst, *(const u32x4*)src);
  } else if constexpr (sizeof(S) == 4) {
    float f[8];
    *(u32x4*)f = *(const u32x4*)src;
    *(u32x4*)(f + 4) = *(const u32x4*)(src + 4);
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      h[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * i], f[2 * i + 1]}, bf16x2));
    store16<LONG>(dst, h);
  } else {
    const uint2 w = *(const uint2*)src;
    store16<LONG>(dst, (u32x4){w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u});
  }
}

// Rows g0, g0 + stride, .. of an append; T, KS, VS: u16 (bf16) or float.
template <bool LONG, typename T, typename KS, typename VS>
__device__ __forceinline__ void append_rows(const PagesK& a, const RowMap& m, const KS* k, const VS* v,
                                            uint32_t g0, uint32_t stride) {
  constexpr int V = 16 / sizeof(T);
  const int d = a.pg.head_dim, cpr = d / V;   // 8, 16 or 32 chunks per row
  const int c = (threadIdx.x & (cpr - 1)) * V, mask = (1 << a.shift) - 1;
  for (uint32_t g = g0; g < m.rows; g += stride) {
    int e, row;
    map_row(m, g, &e, &row);
    const PageJob j = a.jobs[e];
    if (row >= j.n1 - j.n0) continue;   // (a refused entry's n1 is -1)
    const int slot = j.n0 + row, ord = slot >> a.shift;
    int32_t* entry = a.pg.table + (size_t)j.dst * a.pg.max_pages + ord;
    int page;
    if (ord < j.first) {
      page = *entry;
      if ((unsigned)page >= (unsigned)a.pg.pages) continue;
    } else {
      page = a.ids[j.off + ord - j.first];
      if (c == 0 && (slot & mask) == 0) {
        *entry = page;
        a.pg.refs[page] = 1;
      }
    }
    const size_t to = (((size_t)page << a.shift) + (slot & mask)) * d + c;
    const size_t from = (size_t)(j.start + row) * d + c;
    copy16<LONG>(k + from, (T*)a.pg.k + to);
    copy16<LONG>(v + from, (T*)a.pg.v + to);
  }
}

template <typename T, typename KS, typename VS>
__global__ __launch_bounds__(kCopyTh) void append_kernel(PagesK a, RowMap m, const KS* k, const VS* v) {
  const int cpr = a.pg.head_dim * (int)sizeof(T) / 16, per = kCopyTh / cpr;
  append_rows<true, T>(a, m, k, v, blockIdx.x * per + threadIdx.x / cpr, gridDim.x * per);
}

// The few rows of a decoding step, by the block that plans them.
template <typename T, typename KS, typename VS>
__global__ __launch_bounds__(kPlanTh) void plan_append_kernel(PagesK a, RowMap m, const KS* k, const VS* v) {
  make_plan_block(a);
  __syncthreads();
  const int cpr = a.pg.head_dim * (int)sizeof(T) / 16;
  append_rows<false, T>(a, m, k, v, threadIdx.x / cpr, kPlanTh / cpr);
}

// The slot of row `row` behind the first `first` rows of a unit that has n1 after the call
// (-1 where it is refused), or -1.  `row` may come near 2^31, as a call's rows are only a bound
// on its counts, so it is compared before it is added.
__device__ __forceinline__ int new_slot(int first, int row, int n1) {
  return row < n1 - first ? first + row : -1;
}

// Slot `row` of the new pages of a fork or a compaction, read through the old
// table; this thread's 16 bytes of K and V at column c.
template <typename T>
__device__ __forceinline__ void move_row(const PagesK& a, const PageJob& j, int e, int row, int c,
                                         const int32_t* idx) {
  const int d = a.pg.head_dim, mask = (1 << a.shift) - 1;
  const int slot = new_slot(j.first << a.shift, row, j.n1);
  if (slot < 0) return;
  int from = slot;
  if (slot >= j.keep) from = idx[j.start + (slot - j.keep)];
  u32x4 rk = {0, 0, 0, 0}, rv = rk;
  if ((unsigned)from < (unsigned)j.n0) {
    const int p = a.pg.table[(size_t)j.src * a.pg.max_pages + (from >> a.shift)];
    if ((unsigned)p < (unsigned)a.pg.pages) {
      const size_t at = (((size_t)p << a.shift) + (from & mask)) * d + c;
      rk = *(const u32x4*)((const T*)a.pg.k + at);
      rv = *(const u32x4*)((const T*)a.pg.v + at);
    }
  } else if (c == 0 && a.status) {
    a.status[e] = GRKV_PAGES_RANGE;
  }
  const int page = a.ids[j.off + (slot >> a.shift) - j.first];
  const size_t to = (((size_t)page << a.shift) + (slot & mask)) * d + c;
  store16<true>((T*)a.pg.k + to, rk);
  store16<true>((T*)a.pg.v + to, rv);
}

template <typename T>
__global__ __launch_bounds__(kCopyTh) void move_kernel(PagesK a, RowMap m, const int32_t* idx) {
  constexpr int V = 16 / sizeof(T);
  const int cpr = a.pg.head_dim / V;   // 8, 16 or 32 chunks per row
  const int c = (threadIdx.x & (cpr - 1)) * V;
  const uint32_t stride = gridDim.x * (kCopyTh / cpr);
  for (uint32_t g = blockIdx.x * (kCopyTh / cpr) + threadIdx.x / cpr; g < m.rows; g += stride) {
    int e, row;
    map_row(m, g, &e, &row);
    move_row<T>(a, a.jobs[e], e, row, c, idx);
  }
}

// Page p of each lane (or -1) leaves one table; one that no table holds any more is
// free.  Every lane of the wave takes part: neighbours whose pages share a word of
// the bitmap (a unit's pages mostly follow one another) set their bits by one atomic,
// since all words of a pool lie in few cache lines.  (2048 pages of 8 units by
// one atomic each took 12 us.)
__device__ __forceinline__ void release_pages(const grkv_pages& pg, int p) {
  uint32_t bit = 0;
  int word = -1;
  if ((unsigned)p < (unsigned)pg.pages && atomicSub(pg.refs + p, 1) == 1) {
    word = p >> 5;
    bit = 1u << (p & 31);
  }
  const int lane = threadIdx.x & 63;
  // bits of the run of equal words that ends at this lane
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t b = __shfl_up(bit, k);
    const int w = __shfl_up(word, k);
    if (lane >= k && w == word) bit |= b;
  }
  const int next = __shfl_down(word, 1);
  if (word >= 0 && (lane == 63 || next != word)) atomicOr(pg.free_bits + word, bit);
}

// The destination's table row and the counts, by the threads of a block.  A page
// that is given up here and shared there (two entries, one page) never passes
// zero in between: the unit it is shared from keeps it.
__device__ __forceinline__ void commit(const PagesK& a, const PageJob& j) {
  if (j.n1 < 0) return;
  const int32_t* from = a.pg.table + (size_t)j.src * a.pg.max_pages;
  int32_t* to = a.pg.table + (size_t)j.dst * a.pg.max_pages;
  if (j.src != j.dst) {
    for (int o = threadIdx.x; o < j.first; o += blockDim.x) {
      const int p = from[o];
      to[o] = p;
      if ((unsigned)p < (unsigned)a.pg.pages) atomicAdd(a.pg.refs + p, 1);
    }
  }
  const int held = j.src == j.dst ? (j.n0 + (1 << a.shift) - 1) >> a.shift : 0;
  const int end = max(held, j.last);
  for (int o0 = j.first; o0 < end; o0 += blockDim.x) {
    const int o = o0 + threadIdx.x;
    release_pages(a.pg, o < held ? to[o] : -1);
    if (o >= end) continue;
    int p = -1;
    if (o < j.last) {
      p = a.ids[j.off + o - j.first];
      a.pg.refs[p] = 1;
    }
    to[o] = p;
  }
}

__global__ __launch_bounds__(kCopyTh) void commit_kernel(PagesK a) { commit(a, a.jobs[blockIdx.x]); }

// Both, one block per entry: the rows that are read through the old table row are
// copied before the row changes (no other entry reads it: a unit is not both read
// and written by two entries).
template <typename T>
__global__ __launch_bounds__(kCopyTh) void move_commit_kernel(PagesK a, const int32_t* idx) {
  constexpr int V = 16 / sizeof(T);
  const PageJob j = a.jobs[blockIdx.x];
  const int cpr = a.pg.head_dim / V;
  const int c = (threadIdx.x & (cpr - 1)) * V, rows = j.n1 - (j.first << a.shift);
#pragma unroll 4
  for (int row = threadIdx.x / cpr; row < rows; row += kCopyTh / cpr)
    move_row<T>(a, j, blockIdx.x, row, c, idx);
  __syncthreads();
  commit(a, j);
}

// One block per entry.  The first block to take a unit's length frees it.
__global__ __launch_bounds__(kCopyTh) void free_kernel(PagesK a) {
  __shared__ int n_s;
  const int i = blockIdx.x, u = a.units ? a.units[i] : i;
  const bool ok = (unsigned)u < (unsigned)a.pg.units;
  if (threadIdx.x == 0) {
    if (a.status) a.status[i] = ok ? GRKV_PAGES_OK : GRKV_PAGES_UNIT;
    n_s = ok ? atomicExch(a.pg.lens + u, 0) : 0;
  }
  __syncthreads();
  if (n_s <= 0) return;
  const int held = min((n_s - 1 >> a.shift) + 1, a.pg.max_pages);
  int32_t* row = a.pg.table + (size_t)u * a.pg.max_pages;
  for (int o0 = 0; o0 < held; o0 += kCopyTh) {
    const int o = o0 + threadIdx.x;
    release_pages(a.pg, o < held ? row[o] : -1);
    if (o < held) row[o] = -1;
  }
}

__global__ __launch_bounds__(kCopyTh) void init_kernel(PagesK a) {
  const int64_t stride = (int64_t)gridDim.x * kCopyTh;
  const int64_t at = (int64_t)blockIdx.x * kCopyTh + threadIdx.x;
  for (int64_t i = at; i < (int64_t)a.pg.units * a.pg.max_pages; i += stride) a.pg.table[i] = -1;
  for (int64_t i = at; i < a.pg.units; i += stride) a.pg.lens[i] = 0;
  for (int64_t i = at; i < a.pg.pages; i += stride) a.pg.refs[i] = 0;
  for (int64_t i = at; i < (a.pg.pages + 31) / 32; i += stride) {
    const int64_t left = a.pg.pages - 32 * i;
    a.pg.free_bits[i] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
  }
}

PagesK make_args(const PagesCall& c) {
  PagesK a = {};
  a.pg = *c.pages;
  a.shift = __builtin_ctz((unsigned)c.pages->page_size);
  a.op = c.op;
  if (c.entries) {
    a.entries = c.entries->entries;
    a.rows = c.op == kPagesFork ? 0 : c.entries->rows;
    a.units = c.entries->units;
    a.status = c.entries->status;
    if (c.op != kPagesFork) {
      a.counts = c.entries->counts;
      a.starts = c.entries->starts;
      a.source_rows = c.entries->source_rows;
    }
  }
  a.dst = c.dst;
  a.keep = c.keep;
  if (c.workspace) {
    char* ws = (char*)c.workspace;
    const PagesLayout lay = pages_layout(c.pages, a.entries);
    a.owner = (int32_t*)(ws + lay.owner);
    a.jobs = (PageJob*)(ws + lay.jobs);
    a.ids = (int32_t*)(ws + lay.ids);
  }
  return a;
}

// Rows of at most `most` per entry.
RowMap make_map(int entries, int64_t most) {
  RowMap m;
  m.tile_shift = 0;
  while (m.tile_shift < 6 && (1 << m.tile_shift) < most) ++m.tile_shift;
  m.per = (uint32_t)((most + (1 << m.tile_shift) - 1) >> m.tile_shift);
  m.rows = ((uint32_t)entries * m.per) << m.tile_shift;
  return m;
}

// Blocks for that many rows, `per_block` at a time: one step per thread until
// the card is full eight times over, then more steps.
unsigned copy_blocks(const RowMap& m, int per_block) {
  const uint32_t b = (m.rows + per_block - 1) / per_block;
  return b < 16384 ? b : 16384;
}

// Rows of a call that the planning block stores itself (one row for each of 32
// units: one launch of 5.7 us against two of 6.9 and 3.5).
constexpr int64_t kInlineRows = 128;

template <typename T, typename KS, typename VS>
void launch_append(const PagesK& a, const PagesCall& c, hipStream_t s) {
  const RowMap m = make_map(a.entries, a.rows);
  const KS* k = (const KS*)c.k;
  const VS* v = (const VS*)c.v;
  if ((int64_t)a.entries * a.rows <= kInlineRows) {
    hipLaunchKernelGGL((plan_append_kernel<T, KS, VS>), dim3(1), dim3(kPlanTh), 0, s, a, m, k, v);
    return;
  }
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanTh), 0, s, a);
  hipLaunchKernelGGL((append_kernel<T, KS, VS>), dim3(copy_blocks(m, kCopyTh * 16 / (a.pg.head_dim * (int)sizeof(T)))),
                     dim3(kCopyTh), 0, s, a, m, k, v);
}

template <typename T>
void launch_append_t(const PagesK& a, const PagesCall& c, hipStream_t s) {
  if (c.k_dtype == GRKV_BF16)
    c.v_dtype == GRKV_BF16 ? launch_append<T, u16, u16>(a, c, s) : launch_append<T, u16, float>(a, c, s);
  else
    c.v_dtype == GRKV_BF16 ? launch_append<T, float, u16>(a, c, s) : launch_append<T, float, float>(a, c, s);
}

// Fork and compact.  An entry of up to kEntryRows rows (those under keep in its page,
// then the picked ones), or one of very many, is one block's; longer ones are
// spread over blocks and committed by a launch of their own.
constexpr int64_t kEntryRows = 256, kManyEntries = 512;

template <typename T>
void launch_move(const PagesK& a, const PagesCall& c, hipStream_t s) {
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanTh), 0, s, a);
  const int64_t most = (int64_t)a.rows + (c.op == kPagesFork || c.keep ? a.pg.page_size - 1 : 0);
  if (most <= kEntryRows || a.entries >= kManyEntries) {
    hipLaunchKernelGGL((move_commit_kernel<T>), dim3(a.entries), dim3(kCopyTh), 0, s, a, c.idx);
    return;
  }
  const RowMap m = make_map(a.entries, most);
  hipLaunchKernelGGL((move_kernel<T>), dim3(copy_blocks(m, kCopyTh / (a.pg.head_dim * (int)sizeof(T) / 16))),
                     dim3(kCopyTh), 0, s, a, m, c.idx);
  hipLaunchKernelGGL(commit_kernel, dim3(a.entries), dim3(kCopyTh), 0, s, a);
}

}  // namespace

PagesLayout pages_layout(const grkv_pages* pg, int entries) {
  PagesLayout l;
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  l.owner = 0;
  l.jobs = l.owner + up((size_t)pg->units * sizeof(int32_t));
  l.ids = l.jobs + up((size_t)entries * sizeof(PageJob));
  l.total = l.ids + up((size_t)pg->pages * sizeof(int32_t));
  return l;
}

hipError_t launch_pages(const PagesCall& c, hipStream_t s) {
  const PagesK a = make_args(c);
  if (c.op == kPagesInit) {
    hipLaunchKernelGGL(init_kernel, dim3(1024), dim3(kCopyTh), 0, s, a);
    return hipGetLastError();
  }
  if (a.entries == 0) return hipSuccess;
  if (c.op == kPagesFree) {
    hipLaunchKernelGGL(free_kernel, dim3(a.entries), dim3(kCopyTh), 0, s, a);
    return hipGetLastError();
  }
  const bool bf16 = a.pg.dtype == GRKV_BF16;
  if (c.op == kPagesAppend) bf16 ? launch_append_t<u16>(a, c, s) : launch_append_t<float>(a, c, s);
  else bf16 ? launch_move<u16>(a, c, s) : launch_move<float>(a, c, s);
  return hipGetLastError();
}

}  // namespace grkv
