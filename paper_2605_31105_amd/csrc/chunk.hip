// Attention of a step's new tokens over their units' pages (grkv_chunk_attention): single
// tokens of some sequences beside chunks of others, in one launch.
//
// The sums are those of attend_rows.h and wide_rows.h.  A job is a tile of rows (tokens by heads
// of the group) of one unit: up to 16 rows take the kernel of few rows, whose four waves each
// read keys of their own and which HBM bounds; more, up to 128, the one of many rows,
// whose waves share tiles of 64 keys in LDS and which its products bound.  float32 has jobs of 16 rows.
// How many rows and keys a job has only the device knows, and a batch holds one key beside
// 100k and one row beside 128, so the key tiles of all jobs are put in a row and cut into
// equal parts, one per block, two blocks per compute unit: no block waits for a longer one, and
// blocks of either kind share a compute unit.  Every block adds up all jobs for itself
// (threads a run of jobs each).  A part goes over the ends of jobs; of a part only
// the first and the last job may be partial, and a second launch adds those up, in order.
// Jobs follow one another by sequence, unit and rows, and an XCD's blocks hold neighbouring
// parts, so that its L2 serves the rows of a unit.
#include "attend_rows.h"
#include "wide_rows.h"

namespace grkv {
namespace {

constexpr int kChunkTh = kAtTh;
constexpr int kChunkBlocks = 512, kXcds = 8;
static_assert(kAtTh == kWTh, "one kernel holds both");

// Rows of a job, and of those that the kernel of few rows takes.
template <typename E>
constexpr int kJobShift = sizeof(E) == 2 ? 7 : 4;
constexpr int kFewRows = 16;

// First row tile of sequence b in the row of all sequences' tiles: one tile more than
// its rows fill for each sequence before it, so that no sum over sequences is needed.
template <typename E>
__device__ __forceinline__ int tile_of(const AttendK& a, int b) {
  const int s = min(max(a.starts[b], 0), a.step_tokens);
  return (int)((int64_t)s * a.group >> kJobShift<E>) + b;
}

// Where a job lies: a sequence, a unit of it and rows r0 ...
struct Job {
  int b;         // sequence, -1: none
  int tile, next;   // its first tile, and the next sequence's
};

// The last sequence whose tiles start at tile w or before (-1: none).
template <typename E>
__device__ __forceinline__ int find_sequence(const AttendK& a, int w) {
  int lo = 0, hi = a.sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (tile_of<E>(a, mid) <= w) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// A job's shape.
struct Shape {
  int b, h, start, t, r0, rows, len;
  const int32_t* trow;
};

// Job j of sequence b, whose tiles are tile .. next - 1; false where there are no rows.
template <typename E>
__device__ __forceinline__ bool shape_of(const AttendK& a, int64_t j, int b, int tile, int next, Shape* s) {
  const int n = next - tile;
  const int64_t local = j - (int64_t)tile * a.heads;
  if (b < 0 || n < 1 || local < 0 || local >= (int64_t)n * a.heads) return false;   // (starts that fall)
  s->b = b;
  s->h = (int)((uint32_t)local / (uint32_t)n);
  s->start = min(max(a.starts[b], 0), a.step_tokens);
  s->t = min(min(max(a.starts[b + 1], 0), a.step_tokens) - s->start, a.longest);
  s->r0 = ((int)local - s->h * n) << kJobShift<E>;
  const int64_t R = (int64_t)s->t * a.group;
  if (s->r0 >= R) return false;
  s->rows = (int)(R - s->r0 < (1 << kJobShift<E>) ? R - s->r0 : 1 << kJobShift<E>);
  const int u = a.units ? a.units[b * a.unit_stride + s->h] : b * a.heads + s->h;
  const bool ok = (unsigned)u < (unsigned)a.pool_units;
  s->len = ok ? min(max(a.lens[u], 0), a.max_pages << a.shift) : 0;
  s->trow = a.table + (size_t)(ok ? u : 0) * a.max_pages;
  return true;
}

template <typename E>
__device__ __forceinline__ bool few(const Shape& s) {
  return sizeof(E) == 4 || s.rows <= kFewRows;
}

template <typename E>
__device__ __forceinline__ Span span_of(const AttendK& a, const Shape& s) {
  return make_span(a, false, s.len, s.len - s.t, s.t, group_of(a, s.r0), group_of(a, s.r0 + s.rows - 1),
                   few<E>(s) ? Tile<E>::KEYS : kWideKeys);
}

// The tiles of a job as parts count them: one at least, so that a job without keys is some
// block's too; 0 without rows.
template <typename E>
__device__ __forceinline__ int job_tiles(const AttendK& a, int64_t j, int b, int tile, int next) {
  Shape s;
  if (!shape_of<E>(a, j, b, tile, next, &s)) return 0;
  return max(span_of<E>(a, s).nt, 1);
}

// A walk over jobs in order, which keeps the sequence it is in.
template <typename E>
struct Walk {
  int b, tile, next;
  int64_t end;    // first job behind the sequence
  __device__ __forceinline__ void enter(const AttendK& a, int to) {
    b = to;
    tile = b >= 0 ? tile_of<E>(a, b) : 0;
    next = b + 1 <= a.sequences ? tile_of<E>(a, b + 1) : tile;
    end = (int64_t)next * a.heads;
  }
  __device__ __forceinline__ void start(const AttendK& a, int64_t j) {
    enter(a, min(find_sequence<E>(a, (int)(j / a.heads)), a.sequences - 1));
  }
  __device__ __forceinline__ void to(const AttendK& a, int64_t j) {
    while (j >= end && b + 1 < a.sequences) enter(a, b + 1);
  }
};

template <typename E, int D>
__global__ __launch_bounds__(kChunkTh, 2) void chunk_kernel(AttendK a) {
  constexpr int BYTES = kStage<E, D>;
  static_assert(sizeof(E) == 4 || BYTES == kRing<D>, "both kinds take the same LDS");
  __shared__ __attribute__((aligned(1024))) char v0_s[BYTES];
  __shared__ __attribute__((aligned(1024))) char v1_s[BYTES];
  __shared__ int64_t sum_s[kChunkTh / 64];
  __shared__ int64_t at_s, first_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t blocks = gridDim.x, b = (blockIdx.x % kXcds) * (blocks / kXcds) + blockIdx.x / kXcds;

  // tiles before this thread's jobs, and of all
  const int64_t per = (a.jobs + kChunkTh - 1) / kChunkTh;
  const int64_t j0 = tid * per, j1 = j0 + per < a.jobs ? j0 + per : a.jobs;
  int64_t own = 0;
  Walk<E> w;
  if (j0 < j1) {
    w.start(a, j0);
    for (int64_t j = j0; j < j1; ++j) {
      w.to(a, j);
      own += job_tiles<E>(a, j, w.b, w.tile, w.next);
    }
  }
  int64_t incl = own;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t x = __shfl_up((long long)incl, k);
    if (lane >= k) incl += x;
  }
  if (lane == 63) sum_s[wave] = incl;
  __syncthreads();
  int64_t all = 0, at = incl - own;
#pragma unroll
  for (int k = 0; k < kChunkTh / 64; ++k) {
    if (k < wave) at += sum_s[k];
    all += sum_s[k];
  }
  all = uniform64(all);
  const int64_t part = max((int64_t)a.min_tiles, (all + blocks - 1) / blocks);
  const int64_t lo = b * part, hi = min(all, lo + part);
  if (tid == 0) a.ends[b] = make_int4(-1, 0, 0, 0);
  if (lo >= all) return;
  if (at <= lo && lo < at + own) {   // this thread's: the job of the part's first tile
    int64_t j = j0;
    w.start(a, j);
    for (; j < j1; ++j) {
      w.to(a, j);
      const int n = job_tiles<E>(a, j, w.b, w.tile, w.next);
      if (lo < at + n) break;
      at += n;
    }
    first_s = j;
    at_s = at;
  }
  __syncthreads();
  int64_t from = uniform64(at_s), j = uniform64(first_s);
  w.start(a, j);
  for (; from < hi && j < a.jobs; ++j) {
    w.to(a, j);
    Shape s;
    if (!shape_of<E>(a, j, __builtin_amdgcn_readfirstlane(w.b), __builtin_amdgcn_readfirstlane(w.tile),
                     __builtin_amdgcn_readfirstlane(w.next), &s))
      continue;
    AttendK x = a;   // the unit's own rows
    const size_t row0 = (size_t)s.start * a.q_heads + (size_t)s.h * a.group;
    x.q = (const E*)a.q + row0 * D;
    x.o = (E*)a.o + row0 * D;
    x.lse = a.lse ? a.lse + row0 : nullptr;
    x.tokens = s.t;
    x.row_groups = (int64_t)s.t * a.group <= 1 << kJobShift<E> ? 1 : 2;   // (one or more)
    const Span sn = span_of<E>(a, s);
    const int64_t to = from + max(sn.nt, 1);
    const int vt0 = (int)(max(lo, from) - from), vt1 = min((int)(min(hi, to) - from), sn.nt);
    const bool whole = from >= lo && to <= hi;
    const int64_t slot = 2 * b + (from > lo ? 1 : 0);
    const int64_t rows_at = slot * a.part_rows - s.r0;   // partial row of row r: this + r
    if (from >= lo && !whole && tid == 0)
      a.ends[b] = make_int4((int)j, (int)(min((to - 1) / part, blocks - 1) - b) + 1, (int)(slot & 1), 0);
    if (few<E>(s)) {
      attend_rows<E, D, 1, kChunk>(x, sn, 0, s.r0, vt0, vt1, whole ? kWhole : rows_at, false, s.len, s.t, s.trow,
                                   v0_s, v1_s);
    } else if constexpr (sizeof(E) == 2) {
      wide_rows<D, kChunk>(x, sn, 0, s.r0, vt0, vt1, [&] { return Part{!whole, rows_at}; }, s.len, s.t, s.trow,
                           v0_s, v1_s);
    }
    __syncthreads();   // (the next rows take the same stages)
    from = to;
  }
}

// The rows of jobs that were cut: those that began in part blockIdx.x, 16 rows a block.
template <typename E, int D>
__global__ __launch_bounds__(kChunkTh) void chunk_combine_kernel(AttendK a) {
  constexpr int CR = D / 4;
  const int4 p = a.ends[blockIdx.x];
  if (p.x < 0 || p.y < 2) return;
  Walk<E> w;
  w.start(a, p.x);
  Shape s;
  if (!shape_of<E>(a, p.x, w.b, w.tile, w.next, &s)) return;
  const int first = 16 * blockIdx.y;
  const size_t row0 = (size_t)s.start * a.q_heads + (size_t)s.h * a.group;
  AttendK x = a;
  x.o = (E*)a.o + row0 * D;
  x.lse = a.lse ? a.lse + row0 : nullptr;
  for (int c = threadIdx.x; c < 16 * CR; c += kChunkTh) {
    const int row = first + c / CR, ch = c % CR;
    if (row >= s.rows) continue;
    const int r = s.r0 + row, i = group_of(a, r), g = r - i * a.group;
    const Split o = add_splits<D, false>(a, (size_t)2 * blockIdx.x * a.part_rows + row, p.z * a.part_rows,
                                         2 * a.part_rows, p.y, 0, 1, ch);
    write_out<E, D>(x, row_at<kChunk>(x, 0, g, i), ch, o.x, o.m, o.l, o.lx);
  }
}

template <typename E, int D>
hipError_t launch_ed(const AttendK& a, hipStream_t s) {
  hipLaunchKernelGGL((chunk_kernel<E, D>), dim3((unsigned)a.blocks), dim3(kChunkTh), 0, s, a);
  hipLaunchKernelGGL((chunk_combine_kernel<E, D>), dim3((unsigned)a.blocks, (a.part_rows + 15) / 16),
                     dim3(kChunkTh), 0, s, a);
  return hipGetLastError();
}

}  // namespace

ChunkPlan chunk_plan(const grkv_step* step, const grkv_chunk* ch, int d, int dtype, int64_t slots) {
  ChunkPlan p;
  const int shift = dtype == GRKV_BF16 ? kJobShift<u16> : kJobShift<float>;
  p.jobs = (((int64_t)step->tokens * ch->group >> shift) + step->sequences) * step->heads;
  p.min_part = 8;   // (two tiles for each wave of a block of few rows)
  const int64_t rows = (int64_t)(ch->longest < step->tokens ? ch->longest : step->tokens) * ch->group;
  p.part_rows = rows >= 1 << shift ? 1 << shift : rows > 16 ? (int)((rows + 15) / 16 * 16) : 16;
  // parts of the longest units, if all are
  const int64_t keys = dtype == GRKV_BF16 ? Tile<u16>::KEYS : Tile<float>::KEYS;
  const int64_t parts = ((slots + keys - 1) / keys + p.min_part - 1) / p.min_part;
  int64_t blocks = p.jobs < kChunkBlocks ? p.jobs * (parts < kChunkBlocks ? parts : kChunkBlocks) : kChunkBlocks;
  blocks = blocks < kChunkBlocks ? (blocks + kXcds - 1) / kXcds * kXcds : kChunkBlocks;
  p.blocks = (int)(blocks > kXcds ? blocks : kXcds);
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  const size_t part = 2 * (size_t)p.blocks * p.part_rows;
  p.opart = 0;
  p.mpart = up(part * d * sizeof(float));
  p.ends = p.mpart + up(part * sizeof(float4));
  p.total = p.ends + up((size_t)p.blocks * sizeof(int4));
  return p;
}

hipError_t launch_chunk(AttendK a, const ChunkPlan& p, int d, int dtype, void* workspace, hipStream_t s) {
  a.splits = 1;
  a.split_shift = 0;
  a.min_tiles = p.min_part;
  a.blocks = p.blocks;
  a.jobs = p.jobs;
  a.part_rows = p.part_rows;
  a.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)d));
  a.opart = (float*)((char*)workspace + p.opart);
  a.mpart = (float4*)((char*)workspace + p.mpart);
  a.ends = (int4*)((char*)workspace + p.ends);
  set_group(a);
  if (dtype == GRKV_BF16) return d == 64 ? launch_ed<u16, 64>(a, s) : launch_ed<u16, 128>(a, s);
  return d == 64 ? launch_ed<float, 64>(a, s) : launch_ed<float, 128>(a, s);
}

}  // namespace grkv
