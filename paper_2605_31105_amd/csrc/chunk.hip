// Attention of a step's new tokens over their units' pages (grkv_chunk_attention): single
// tokens of some sequences beside chunks of others, in one launch.
//
// The sums are those of attend_rows.h and wide_rows.h.  A job is a tile of rows (tokens by heads
// of the group) of one unit: up to 16 rows take the kernel of few rows, whose four waves each
// read keys of their own and which HBM bounds; more, up to 128, the one of many rows,
// whose waves share tiles of 64 keys in LDS and which its exponentials and products bound.
// float32 has jobs of 32 rows, by the kernel of few rows.  Calls without longer sequences than one
// or two 16-row tiles have kernels of their own, with the code of few rows alone.
// How many rows and keys a job has only the device knows, and a batch holds one key beside
// 100k and one row beside 128, so the costs of all jobs are put in a row and cut into equal
// parts, one per block, two blocks per compute unit: no block waits for a longer one, and
// blocks of either kind share a compute unit.  Every block adds up all jobs for itself
// (threads a run of jobs each).  A part goes over the ends of jobs; of a part only
// the first and the last job may be partial, and a second launch adds those up, in order.
// Jobs follow one another by sequence, unit and rows, and an XCD's blocks hold neighbouring
// parts, so that its L2 serves the rows of a unit (51% of reads, 21% where whole jobs did not
// come first).
//
// Measured (bf16, 8 KV heads of 128 columns, 4 query heads each): a token of 64 sequences of 500 to
// 8000 keys 195 us (1.11 GB, 5.7 TB/s); beside two chunks of 512, 275; four chunks of 2048 over 4k to
// 14k 1320 to 1350 (1.0 PFLOP/s, the clock at 1.8 GHz); one token over 2048 keys 16.5, a chain of reads.
#include "attend_rows.h"
#include "wide_rows.h"

namespace grkv {
namespace {

constexpr int kChunkTh = kAtTh;
constexpr int kChunkBlocks = 512, kXcds = 8;
static_assert(kAtTh == kWTh, "one kernel holds both");

// Rows of a job, and of those that the kernel of few rows takes.
template <typename E>
constexpr int kJobShift = sizeof(E) == 2 ? 7 : 5;
constexpr int kFewRows = 16;
// Jobs of so many rows have weights of two bf16 parts in the kernel of many rows too (2^-15 of a weight,
// as a tree of as many rows has): their keys' bytes bound them, and a sequence of up to 64 rows has them
// as exact whatever others the call holds.  (16 tokens of 64 sequences of 500 to 8000 keys, 64 rows
// a unit: 257 us with rounded weights and two waves without rows, 254 so.  Longer jobs are bound by their products: see
// attend_wide.hip.)
constexpr int kTwoParts = 64;
// Costs, in half tiles of 32 keys read for few rows (kTwo: two
// 16-row tiles of them, 32 keys of bf16 or 16 of float32).
// Timed blocks take 1.05 us for such a tile, 2.4 to 2.8 for 64 keys of many rows and some two
// tiles more for a job's first reads and its outputs; a token of 64 sequences beside two chunks of
// 512 with the latter tile at 4, 5 and 6: 285, 272 and 282 us.
constexpr int kFewFixed = 6, kFewTile = 2, kWideFixed = 15, kWideTile = 5, kTwoFixed = 9, kTwoTile = 3;
// Calls of so few jobs give every block a piece of one job, and pieces of few rows, up to kJoined
// of a job, are joined by the block that ends last (8 units of 2048 keys and one token, both
// together 22 -> 17 us).
constexpr int kAlignedJobs = 64, kJoined = 16;
// Jobs of a thread whose lengths are read together (66 sequences, 784 jobs: a call of 274 -> 272
// us).
constexpr int kTogether = 4;
// Starts that a block keeps in LDS, where the searches of its threads read them.
constexpr int kStartsHeld = 1024;

// First row tile of sequence b in the row of all sequences' tiles: one tile more than
// its rows fill for each sequence before it, so that no sum over sequences is needed.
template <typename E>
__device__ __forceinline__ int tile_of(const AttendK& a, const int32_t* starts, int b) {
  const int s = min(max(starts[b], 0), a.step_tokens);
  return (int)((int64_t)s * a.group >> kJobShift<E>) + b;
}

// The last sequence whose tiles start at tile w or before (-1: none).
template <typename E>
__device__ __forceinline__ int find_sequence(const AttendK& a, const int32_t* starts, int w) {
  int lo = 0, hi = a.sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (tile_of<E>(a, starts, mid) <= w) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// A job's shape.
struct Shape {
  int h, start, t, r0, rows, unit, len;   // unit -1: outside the pool
  const int32_t* trow;
  __device__ __forceinline__ void hold() {   // (see Walk)
    for (int* x : {&h, &start, &t, &r0, &rows, &unit}) *x = __builtin_amdgcn_readfirstlane(*x);
  }
};

// Job j of sequence b, whose tiles are tile .. next - 1; false where there are no rows.
template <typename E>
__device__ __forceinline__ bool shape_of(const AttendK& a, const int32_t* starts, int64_t j, int b, int tile, int next,
                                         Shape* s) {
  const int n = next - tile;
  const int64_t local = j - (int64_t)tile * a.heads;
  if (b < 0 || n < 1 || local < 0 || local >= (int64_t)n * a.heads) return false;   // (starts that fall)
  s->h = (int)((uint32_t)local / (uint32_t)n);
  s->start = min(max(starts[b], 0), a.step_tokens);
  s->t = min(min(max(starts[b + 1], 0), a.step_tokens) - s->start, a.longest);
  s->r0 = ((int)local - s->h * n) << kJobShift<E>;
  const int64_t R = (int64_t)s->t * a.group;
  if (s->r0 >= R) return false;
  s->rows = (int)(R - s->r0 < (1 << kJobShift<E>) ? R - s->r0 : 1 << kJobShift<E>);
  const int u = a.units ? a.units[b * a.unit_stride + s->h] : b * a.heads + s->h;
  s->unit = (unsigned)u < (unsigned)a.pool_units ? u : -1;
  return true;
}
__device__ __forceinline__ int raw_len(const AttendK& a, const Shape& s) { return s.unit >= 0 ? a.lens[s.unit] : 0; }
__device__ __forceinline__ void set_len(const AttendK& a, int len, Shape* s) {
  s->len = min(max(len, 0), a.max_pages << a.shift);
  s->trow = a.table + (size_t)max(s->unit, 0) * a.max_pages;
}

__device__ __forceinline__ bool few(const Shape& s) { return s.rows <= kFewRows; }

template <typename E>
__device__ __forceinline__ Span span_of(const AttendK& a, const Shape& s) {
  return make_span(a, false, s.len, s.len - s.t, s.t, group_of(a, s.r0), group_of(a, s.r0 + s.rows - 1),
                   sizeof(E) == 4 || a.rt == 2 || few(s) ? Tile<E>::KEYS : kWideKeys);
}

// What jobs cost: `fixed` for the rows themselves, then `tile` for each of `n` tiles (one at
// least, so that a job without keys is some block's too).
struct Cost {
  int fixed, tile, n;
  __device__ __forceinline__ int all() const { return fixed + tile * n; }
  // Tiles before a cut `at` this far into the job.  A cut among the fixed costs lies before the job.
  __device__ __forceinline__ int tiles(int64_t at) const {
    if (at <= fixed) return 0;
    const int64_t t = (at - fixed + tile - 1) / tile;
    return t < n ? (int)t : n;
  }
};
template <typename E>
__device__ __forceinline__ Cost cost_of(const AttendK& a, const Shape& s, const Span& sn) {
  const int n = max(sn.nt, 1);
  return few(s) ? Cost{kFewFixed, kFewTile, n}
         : sizeof(E) == 4 || a.rt == 2 ? Cost{kTwoFixed, kTwoTile, n} : Cost{kWideFixed, kWideTile, n};
}

// A walk over jobs in order, which keeps the sequence it is in.
template <typename E>
struct Walk {
  const int32_t* starts;
  int b, tile, next;
  int64_t end;    // first job behind the sequence
  __device__ __forceinline__ void enter(const AttendK& a, int to) {
    b = to;
    tile = b >= 0 ? tile_of<E>(a, starts, b) : 0;
    next = b + 1 <= a.sequences ? tile_of<E>(a, starts, b + 1) : tile;
    end = (int64_t)next * a.heads;
  }
  __device__ __forceinline__ void start(const AttendK& a, int64_t j) {
    enter(a, min(find_sequence<E>(a, starts, (int)((uint32_t)j / (uint32_t)a.heads)), a.sequences - 1));
  }
  __device__ __forceinline__ void to(const AttendK& a, int64_t j) {
    while (j >= end && b + 1 < a.sequences) enter(a, b + 1);
  }
  // (the same in all lanes: kept in scalar registers)
  __device__ __forceinline__ void hold() {
    b = __builtin_amdgcn_readfirstlane(b);
    tile = __builtin_amdgcn_readfirstlane(tile);
    next = __builtin_amdgcn_readfirstlane(next);
    end = uniform64(end);
  }
};

// Four values of a cut job's row, from its parts in blocks b ..  (JOINED: parts of blocks of this
// launch.)
template <typename E, int D, bool JOINED>
__device__ __forceinline__ void combine_row(const AttendK& a, const CutJob& cut, int64_t b, int row, int ch) {
  if (row >= cut.rows) return;
  AttendK x = a;
  x.o = (E*)a.o + cut.row0 * D;
  x.lse = a.lse ? a.lse + cut.row0 : nullptr;
  const int r = cut.r0 + row, i = group_of(a, r), g = r - i * a.group;
  const Split o = add_splits<D, JOINED>(a, (size_t)2 * b * a.part_rows + row, a.part_rows, 2 * a.part_rows,
                                        cut.parts, 0, 1, ch);
  write_out<E, D>(x, row_at<kChunk>(x, 0, g, i), ch, o.x, o.m, o.l, o.lx);
}

// The kernel's arguments, read anew.  A job takes them this way, so that those of the plan and of the
// jobs before are not held over it: the loop over its tiles needs the scalar registers, and what they do
// not hold is kept in lanes of vector registers (scalars read back in two steps of many rows 19 -> 0; 4 chunks
// of 2048 over 4k to 14k 1357 -> 1336 us, 2 of 512 124 -> 117, 4 prompts of 4096 with 64 columns 469 -> 465).
__device__ __forceinline__ AttendK arguments() {
  auto at = __builtin_amdgcn_kernarg_segment_ptr();   // (the first argument lies there)
  asm volatile("" : "+s"(at));
  return *(const AttendK*)at;
}

// RT: 16-row tiles that no job has more of (1, or 2 over bf16 values), 0: rows of any number.
// Jobs of 17 to 32 rows alone are bound by HBM, which the kernel of few rows serves better (64
// sequences of 500 to 8000 keys, 5 tokens of 4 heads each: 235 -> 211 us, one block for each compute
// unit, whose registers hold no second of 128 columns; two in turn 227).
template <typename E, int D, int RT>
__global__ __launch_bounds__(kChunkTh, RT == 2 && D == 128 ? 1 : 2) void chunk_kernel(AttendK a) {
  constexpr bool FEW = RT == 1;   // no job has more than kFewRows rows
  constexpr int BYTES = kStage<E, D>;
  static_assert(sizeof(E) == 4 || BYTES == kRing<D>, "both kinds take the same LDS");
  __shared__ __attribute__((aligned(1024))) char v0_s[BYTES];
  __shared__ __attribute__((aligned(1024))) char v1_s[BYTES];
  __shared__ int64_t sum_s[kChunkTh / 64];
  __shared__ int64_t at_s, first_s;
  __shared__ int pieces_s;
  __shared__ int32_t starts_s[kStartsHeld];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t blocks = gridDim.x, b = (blockIdx.x % kXcds) * (blocks / kXcds) + blockIdx.x / kXcds;

  // This block's part: costs lo .. hi - 1 of all jobs' costs in a row.  Each thread adds up the
  // costs of a run of jobs; the one that has lo's job says where it begins.
  int64_t part = 0, lo = 0, hi = 0;
  auto plan = [&](const int32_t* starts) __attribute__((always_inline)) {
    const int64_t per = (a.jobs + kChunkTh - 1) / kChunkTh;
    const int64_t j0 = tid * per, j1 = min(j0 + per, a.jobs);
    int64_t own = 0;
    int costs[kTogether];   // of the last jobs
    Walk<E> w{starts};
    // the costs of jobs j ..: their reads go out together
    auto together = [&](int64_t j) __attribute__((always_inline)) {
      Shape s[kTogether];
      int len[kTogether];
      bool on[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        on[k] = j + k < j1;
        if (on[k]) {
          w.to(a, j + k);
          on[k] = shape_of<E>(a, starts, j + k, w.b, w.tile, w.next, s + k);
        }
        len[k] = on[k] ? raw_len(a, s[k]) : 0;
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        costs[k] = 0;
        if (!on[k]) continue;
        set_len(a, len[k], s + k);
        costs[k] = cost_of<E>(a, s[k], span_of<E>(a, s[k])).all();
      }
    };
    if (j0 < j1) {
      w.start(a, j0);
      for (int64_t j = j0; j < j1; j += kTogether) {
        together(j);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) own += costs[k];
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
    if (a.aligned) {
      // (a job a thread) blocks of each job by what a part is to cost at most: the least, or so
      // much that all jobs' blocks are there
      auto blocks_for = [&](int64_t cost) {
        const int k = (int)((own + cost - 1) / cost);
        return a.flags ? min(k, kJoined) : k;
      };
      auto scan = [&](int k, int* total) {
        int incl = k;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int x = __shfl_up(incl, d);
          if (lane >= d) incl += x;
        }
        *total = __shfl(incl, 63);
        return incl - k;
      };
      if (wave == 0) {   // (kAlignedJobs at most)
        int total, k = blocks_for(a.min_tiles), first = scan(k, &total);
        if (total > blocks) {
          k = blocks_for(max((int64_t)a.min_tiles, (all + blocks - a.jobs - 1) / (blocks - a.jobs)));
          first = scan(k, &total);
        }
        if (lane == 0) pieces_s = 0;
        if (first <= b && b < first + k) {
          first_s = lane;
          at_s = b - first;
          pieces_s = k;
        }
      }
      return;
    }
    part = max((int64_t)a.min_tiles, (all + blocks - 1) / blocks);
    lo = b * part;
    hi = min(all, lo + part);
    if (at <= lo && lo < at + own) {
      int64_t j = j0;
      if (per > kTogether) w.start(a, j);
      for (bool found = false; !found && j < j1;) {
        if (per > kTogether) together(j);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
          if (found || lo < at + costs[k]) {
            found = true;
          } else {
            at += costs[k];
            ++j;
          }
        }
      }
      first_s = j;
      at_s = at;
    }
  };
  if (a.sequences < kStartsHeld) {
    for (int k = tid; k <= a.sequences; k += kChunkTh) starts_s[k] = a.starts[k];
    __syncthreads();
    plan(starts_s);
  } else {
    plan(a.starts);
  }
  if (tid == 0) a.ends[b].parts = 0;
  if (!a.aligned && lo >= hi) return;
  __syncthreads();
  // this block's piece of its one job
  const int pieces = a.aligned ? __builtin_amdgcn_readfirstlane(pieces_s) : 0;
  if (a.aligned) {
    if (pieces == 0) return;
    hi = 1;
  }
  // whole jobs first: those of a unit, in blocks of one XCD, begin with the same keys at the
  // same time
  for (int pass = 0; pass < 2; ++pass) {
    int64_t from = a.aligned ? 0 : uniform64(at_s), j = uniform64(first_s);
    Walk<E> u{a.starts};
    u.start(a, j);
    for (; from < hi && j < a.jobs; ++j) {
      u.to(a, j);
      u.hold();
      AttendK x = arguments();
      Shape s;
      if (!shape_of<E>(x, x.starts, j, u.b, u.tile, u.next, &s)) continue;
      s.hold();
      set_len(x, __builtin_amdgcn_readfirstlane(raw_len(x, s)), &s);
      const Span sn = span_of<E>(x, s);
      const Cost cost = cost_of<E>(x, s, sn);
      const int64_t at = from;
      int vt0, vt1, parts;
      if (x.aligned) {
        const int i = __builtin_amdgcn_readfirstlane((int)at_s);
        vt0 = (int)((int64_t)cost.n * i / pieces);
        vt1 = (int)((int64_t)cost.n * (i + 1) / pieces);
        parts = pieces;
        from = hi;
      } else {
        vt0 = cost.tiles(lo - at);
        vt1 = cost.tiles(hi - at);
        parts = (int)(min((at + cost.all() - cost.tile) / part, blocks - 1) - b) + 1;   // (the part that ends the job)
        from = at + cost.all();
      }
      const bool whole = vt0 == 0 && vt1 == cost.n;
      if (vt1 <= vt0 || whole != (pass == 0)) continue;
      // the unit's own rows
      void* const o = x.o;
      float* const lse = x.lse;
      const size_t row0 = (size_t)s.start * x.q_heads + (size_t)s.h * x.group;
      x.q = (const E*)x.q + row0 * D;
      x.o = (E*)o + row0 * D;
      x.lse = lse ? lse + row0 : nullptr;
      x.tokens = s.t;
      // a part's two places: what it goes on with, and what it begins and leaves to others
      const int64_t rows_at = (2 * b + (vt0 == 0)) * x.part_rows - s.r0;   // partial row of row r: this + r
      if (vt0 == 0 && !whole && tid == 0) x.ends[b] = {row0, s.r0, s.rows, parts};
      const int end = min(vt1, sn.nt);
      const int64_t to = whole ? kWhole : rows_at;
      if (FEW || few(s)) {
        attend_rows<E, D, 1, kChunk>(x, sn, 0, s.r0, vt0, end, to, FEW && x.flags, s.len, s.t, s.trow, v0_s, v1_s);
      } else if constexpr (!FEW) {
        if constexpr (sizeof(E) == 4 || RT == 2)
          attend_rows<E, D, 2, kChunk>(x, sn, 0, s.r0, vt0, end, to, false, s.len, s.t, s.trow, v0_s, v1_s);
        else if (s.rows <= kTwoParts)
          wide_rows<D, kChunk, true>(x, sn, 0, s.r0, vt0, end, [&] { return Part{!whole, rows_at}; }, s.len, s.t, s.trow,
                                     v0_s, v1_s);
        else
          wide_rows<D, kChunk>(x, sn, 0, s.r0, vt0, end, [&] { return Part{!whole, rows_at}; }, s.len, s.t, s.trow,
                               v0_s, v1_s);
      }
      if constexpr (FEW) {
        const int i = (int)at_s;
        if (x.flags && !whole && splits_done(x, j, i, pieces)) {
          for (int c = tid; c < kFewRows * (D / 4); c += kChunkTh) {
            const CutJob cut = {row0, s.r0, s.rows, pieces};
            AttendK y = x;
            y.o = o;
            y.lse = lse;
            combine_row<E, D, true>(y, cut, b - i, c / (D / 4), c % (D / 4));
          }
        }
      }
      __syncthreads();   // (the next rows take the same stages)
    }
  }
}

// The rows of jobs that were cut: those that began in part blockIdx.x, 16 rows a block.
template <typename E, int D>
__global__ __launch_bounds__(kChunkTh) void chunk_combine_kernel(AttendK a) {
  constexpr int CR = D / 4;
  const CutJob cut = a.ends[blockIdx.x];
  if (cut.parts < 2) return;
  for (int c = threadIdx.x; c < 16 * CR; c += kChunkTh)
    combine_row<E, D, false>(a, cut, blockIdx.x, 16 * blockIdx.y + c / CR, c % CR);
}

template <typename E, int D>
hipError_t launch_ed(const AttendK& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks), th(kChunkTh);
  if (a.rt == 1) {
    hipLaunchKernelGGL((chunk_kernel<E, D, 1>), grid, th, 0, s, a);
  } else if (a.rt == 0) {
    hipLaunchKernelGGL((chunk_kernel<E, D, 0>), grid, th, 0, s, a);
  } else if constexpr (sizeof(E) == 2) {
    hipLaunchKernelGGL((chunk_kernel<E, D, 2>), grid, th, 0, s, a);
  }
  if (!a.flags)
    hipLaunchKernelGGL((chunk_combine_kernel<E, D>), dim3((unsigned)a.blocks, (a.part_rows + 15) / 16), th, 0, s, a);
  return hipGetLastError();
}

}  // namespace

ChunkPlan chunk_plan(const grkv_step* step, const grkv_chunk* ch, int d, int dtype, int64_t slots) {
  ChunkPlan p;
  const int shift = dtype == GRKV_BF16 ? kJobShift<u16> : kJobShift<float>;
  p.jobs = (((int64_t)step->tokens * ch->group >> shift) + step->sequences) * step->heads;
  p.min_part = 8 * kFewTile;   // (two tiles for each wave of a block of few rows)
  const int64_t rows = (int64_t)(ch->longest < step->tokens ? ch->longest : step->tokens) * ch->group;
  p.part_rows = rows >= 1 << shift ? 1 << shift : rows > 16 ? (int)((rows + 15) / 16 * 16) : 16;
  // parts of the longest units, if all are
  const int64_t keys = dtype == GRKV_BF16 ? Tile<u16>::KEYS : Tile<float>::KEYS;
  const int64_t parts = (((slots + keys - 1) / keys) * kFewTile + kFewFixed + p.min_part - 1) / p.min_part;
  p.rt = rows <= kFewRows ? 1 : rows <= 2 * kFewRows && dtype == GRKV_BF16 ? 2 : 0;
  const int most = p.rt == 2 && d == 128 ? kChunkBlocks / 2 : kChunkBlocks;   // (what the card holds at once)
  int64_t blocks = p.jobs < most ? p.jobs * (parts < most ? parts : most) : most;
  p.aligned = p.jobs <= kAlignedJobs;
  if (p.aligned && blocks < 2 * p.jobs) blocks = 2 * p.jobs;
  blocks = blocks < most ? (blocks + kXcds - 1) / kXcds * kXcds : most;
  p.blocks = (int)(blocks > kXcds ? blocks : kXcds);
  p.joined = p.aligned && p.rt == 1 && p.blocks <= kJoined * p.jobs;
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  const size_t part = 2 * (size_t)p.blocks * p.part_rows;
  p.opart = 0;
  p.mpart = up(part * d * sizeof(float));
  p.ends = p.mpart + up(part * sizeof(float4));
  p.flags = p.ends + up((size_t)p.blocks * sizeof(CutJob));
  p.total = p.flags + (p.joined ? up((size_t)p.jobs * kJoined * sizeof(uint64_t)) : 0);
  return p;
}

hipError_t launch_chunk(AttendK a, const ChunkPlan& p, int d, int dtype, void* workspace, hipStream_t s) {
  a.splits = kJoined;   // (of the marks)
  a.split_shift = 0;
  a.rt = p.rt;
  a.aligned = p.aligned;
  a.flags = p.joined ? (uint64_t*)((char*)workspace + p.flags) : nullptr;
  a.nonce = p.joined ? next_nonce() : 0;
  a.min_tiles = p.min_part;
  a.blocks = p.blocks;
  a.jobs = p.jobs;
  a.part_rows = p.part_rows;
  a.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)d));
  a.opart = (float*)((char*)workspace + p.opart);
  a.mpart = (float4*)((char*)workspace + p.mpart);
  a.ends = (CutJob*)((char*)workspace + p.ends);
  set_group(a);
  if (dtype == GRKV_BF16) return d == 64 ? launch_ed<u16, 64>(a, s) : launch_ed<u16, 128>(a, s);
  return d == 64 ? launch_ed<float, 64>(a, s) : launch_ed<float, 128>(a, s);
}

}  // namespace grkv
