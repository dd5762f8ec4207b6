// Attention of a few query rows over many keys: single tokens and trees of
// drafted tokens over the pages of a cache (grkv_tree_attention), and the short
// calls of grkv_sink_attention over contiguous keys.
//
// For every query row r and the slots j that it sees,
//   o_r = sum_j 2^(t_rj - m_r) v_j / sum_j 2^(t_rj - m_r),  t = q . k log2(e) / sqrt(d),
// in one pass over the keys with a running reference m_r.  Rows are the
// (query, head of the group) pairs, query-major, 16 RT per block; a unit's keys
// are split over blocks when there are few units, or all units' keys cut into equal
// parts when their lengths may differ (attend_even_kernel), and over the four waves of
// a block always.  Long calls are bound by HBM: 512 units of 500 to 8000 keys, 1.1 GB in
// 189 us, 6.0 TB/s (6.3 is what a read-only stream reaches); short ones by the chain of
// dependent reads and the launch (8 units of 2048 keys, 11.7 us).
//
//  * A wave walks its own key tiles (32 keys of bf16, 16 of float32) with no
//    barrier: K fragments go from memory to registers in the MFMA A layout and
//    V tiles to LDS (global_load_lds), both one tile ahead of the products, so a
//    compute unit keeps 8 waves x 16 KB in flight (4 with blocks of 32 rows of 128 columns,
//    whose 300 registers and more leave room for one block).
//  * S^T = K Q^T puts a query row in each lane column: the four lanes of a row
//    hold its logits as P^T already lies in the B operand of O^T = V^T P^T (the
//    order of the keys inside a tile is free as long as V^T uses the same), so P
//    never leaves the registers.  V^T comes from the row-major tile by the LDS
//    transpose read.
//  * The reference of a row is set 2^8 above its largest logit and moves only when a
//    logit passes it, so most tiles need no exchange between lanes.  No weight is above 1,
//    so large values (finite ones up to the type's largest) do not overflow the sums.
//  * Over bf16 values P enters the product in two bf16 parts, its upper bits and a rounded
//    rest, so that a weight is off by 2^-15 of it instead of 2^-8: memory bounds these
//    calls, and the second product costs them 0 to 2% (one token over 512 ragged
//    units 187.7 -> 188.8 us, over 8 of 128k 93.2 -> 95.0, 64 units of 32 rows 74.2 -> 74.3,
//    300 of 64 rows 161 -> 161; a rounded upper part takes those two to 76.6 and 170).
//    Both parts are above zero (the rest with 2^-18 of the weight added, which o is divided
//    by too), so an infinity that a row sees stays one.
//  * Tiles that every row sees whole skip the masks.  In the others an entry
//    that a row does not see has weight zero.  An infinity or NaN among the values of
//    such a tile reaches those rows all the same, as NaN (0 x inf); where a sum is
//    NaN and such a tile is the cause, the block does its rows again key by key.  So it does
//    where a row's weights left float32's reach (`far_off`).
// Splits leave (m, sum, O) in float32; combine_kernel adds them in order.
#include "attend_rows.h"

#include <atomic>
#include <chrono>

namespace grkv {
namespace {

// Splits that the blocks themselves join: a few, in calls whose blocks all run at once
// (8 units of 2048 keys and 8 rows, 8 splits: one launch of 11.7 us against 9.8 and 3.9).
// More are combined by a launch of their own, which has more threads for them (256 units
// of 4100 keys, 4 splits: 98 and 5 us against 110), and with several row groups a unit,
// whose splits end at different times, from 16 on (calls of 8 units of 32 rows: 1000 keys,
// 4 splits, 13.7 us joined, 16.6 combined; 4000 keys, 16 splits, 18.4 and 16.5).
constexpr int kJoinedSplits = 16, kJoinedRowSplits = 8, kJoinedBlocks = 512;
// Logits of a call (rows by slots) from which the wide kernel is worth its blocks.
constexpr double kWideLogits = 1 << 20;
// Units of any lengths are cut into equal parts (attend_even_kernel) where a part of the
// longest would have 32 tiles or more (calls of 128 units of 500 to 8000 keys, bf16: 59 us,
// with splits joined 64; 512 units 188, in four splits each 203, in one 228; 64 units of
// 8000 keys, 31 tiles: 55, joined 49), for two blocks per compute unit (512 units: 768 blocks
// 212 us, 1024 194), and up to 4096 units, whose lengths every block reads.
constexpr int kEvenTiles = 32, kEvenBlocks = 512, kEvenEntries = 4096;

template <typename E, int D, int RT, Rows KIND>
__global__ __launch_bounds__(kAtTh, RT == 2 && D == 128 ? 1 : 2) void attend_kernel(AttendK a) {
  __shared__ __attribute__((aligned(16))) char v0_s[kStage<E, D>];
  __shared__ __attribute__((aligned(16))) char v1_s[kStage<E, D>];
  int e, rg, sp;
  if (!block_work(a, &e, &rg, &sp)) return;
  const int R = a.group * a.tokens, r0 = rg * 16 * RT;
  int len, t;
  const int32_t* trow;
  entry_shape(a, e, &len, &t, &trow);
  const Span sn = make_span(a, KIND == kTree, len, len - t, t, group_of(a, r0),
                            group_of(a, min(r0 + 16 * RT - 1, R - 1)), Tile<E>::KEYS);
  const int vt0 = sp * sn.chunk, vt1 = min(sn.nt, vt0 + sn.chunk);
  if (sp > 0 && vt0 >= sn.nt) return;
  attend_rows<E, D, RT, KIND>(a, sn, e, r0, vt0, vt1, sn.ns > 1 ? ((int64_t)e * a.splits + sp) * R : kWhole,
                              a.flags != nullptr, len, t, trow, v0_s, v1_s);

  // the splits of a short call, by the block that finishes last
  if (sn.ns < 2 || !a.flags || !splits_done(a, (size_t)e * a.row_groups + rg, sp, sn.ns)) return;
  constexpr int CR = D / 4;
  for (int c = threadIdx.x; c < 16 * RT * CR; c += kAtTh) {
    const int r = r0 + c / CR, ch = c % CR;
    const int i = group_of(a, r), g = r - i * a.group;
    if (r >= R || i >= t) continue;
    const Split o = add_splits<D, true>(a, (size_t)e * a.splits * R + r, 0, R, sn.ns, 0, 1, ch);
    write_out<E, D>(a, ((size_t)e * a.group + g) * a.tokens + i, ch, o.x, o.m, o.l, o.lx);
  }
}

// The tiles of an entry, as attend_even_kernel counts them: one at least, so that an
// entry without keys is some block's too.
template <typename E, int RT>
__device__ __forceinline__ Span even_span(const AttendK& a, int len, int t, int* tiles) {
  const int R = a.group * a.tokens;
  const Span sn = make_span(a, true, len, len - t, t, 0, group_of(a, min(16 * RT - 1, R - 1)), Tile<E>::KEYS);
  *tiles = max(sn.nt, 1);
  return sn;
}

// Units of any lengths, one row group each: the tiles of all of them in a row, cut into
// as many equal parts as there are blocks, so that no block waits for a longer one.  A
// part goes over the ends of units; of the rows of a part only the first and the last
// unit's may be partial.  Every block adds up the lengths for itself.
template <typename E, int D, int RT>
__global__ __launch_bounds__(kAtTh, RT == 2 && D == 128 ? 1 : 2) void attend_even_kernel(AttendK a) {
  __shared__ __attribute__((aligned(16))) char v0_s[kStage<E, D>];
  __shared__ __attribute__((aligned(16))) char v1_s[kStage<E, D>];
  __shared__ int64_t sum_s[kAtWaves];
  __shared__ int64_t at_s;
  __shared__ int first_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, R = a.group * a.tokens;
  // tiles before this thread's entries, and of all
  const int per = (a.entries + kAtTh - 1) / kAtTh, e0 = tid * per, e1 = min(a.entries, e0 + per);
  int len, t, tiles;
  const int32_t* trow;
  int64_t own = 0;
  for (int e = e0; e < e1; ++e) {
    entry_shape(a, e, &len, &t, &trow);
    even_span<E, RT>(a, len, t, &tiles);
    own += tiles;
  }
  int64_t incl = own;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t b = __shfl_up((long long)incl, k);
    if (lane >= k) incl += b;
  }
  if (lane == 63) sum_s[wave] = incl;
  __syncthreads();
  int64_t all = 0, at = incl - own;
#pragma unroll
  for (int w = 0; w < kAtWaves; ++w) {
    if (w < wave) at += sum_s[w];
    all += sum_s[w];
  }
  all = uniform64(all);
  const int64_t blocks = gridDim.x, b = blockIdx.x;
  const int64_t part = max((int64_t)a.min_tiles, (all + blocks - 1) / blocks);
  const int64_t lo = b * part, hi = min(all, lo + part);
  if (lo >= all) return;
  if (at <= lo && lo < at + own) {   // this thread's: the entry of the part's first tile
    int e = e0;
    for (;; ++e) {
      entry_shape(a, e, &len, &t, &trow);
      even_span<E, RT>(a, len, t, &tiles);
      if (lo < at + tiles) break;
      at += tiles;
    }
    first_s = e;
    at_s = at;
  }
  __syncthreads();
  int64_t from = uniform64(at_s);
  for (int e = __builtin_amdgcn_readfirstlane(first_s); from < hi; ++e) {
    entry_shape(a, e, &len, &t, &trow);
    const Span sn = even_span<E, RT>(a, len, t, &tiles);
    const int64_t to = from + __builtin_amdgcn_readfirstlane(tiles);
    const int vt0 = (int)(max(lo, from) - from), vt1 = (int)(min(hi, to) - from);
    const bool whole = from >= lo && to <= hi;
    const int64_t slot = 2 * b + (from > lo ? 1 : 0);
    if (from >= lo && tid == 0) a.even[e] = make_int2((int)slot, whole ? 1 : (int)((to - 1) / part - b) + 1);
    attend_rows<E, D, RT, kTree>(a, sn, e, 0, vt0, min(vt1, sn.nt), whole ? kWhole : slot * R, false, len, t, trow,
                                 v0_s, v1_s);
    __syncthreads();   // (the next rows take the same stages)
    from = to;
  }
}

// The splits of a row, where they are not joined by attend_kernel: one thread per 4
// values and every GS-th split, whose sums are added in order.  GS: threads that share
// a value.
template <typename E, int D, int GS>
__global__ __launch_bounds__(kAtTh) void combine_kernel(AttendK a) {
  constexpr int CR = D / 4, ROWS = kAtTh / (CR * GS);   // rows of a block
  __shared__ f32x4 part[GS > 1 ? kAtTh : 1];
  __shared__ float psum[3][GS > 1 ? kAtTh : 1];
  const int R = a.group * a.tokens, tid = threadIdx.x;
  const int ch = tid % CR, gs = tid / CR % GS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + tid / (CR * GS);
  const int e = (int)(row / R), r = (int)(row % R);
  bool on = e < a.entries;
  int len = 0, t = 0;
  const int32_t* trow;
  if (on) entry_shape(a, e, &len, &t, &trow);
  const int i = group_of(a, r), g = r - i * a.group;
  int ns = 0, first = 0, stride = R;
  size_t at0 = (size_t)e * a.splits * R + r;
  if (on && i < t && a.even) {
    const int2 p = a.even[e];   // the first part, which may be its block's second
    ns = p.y;
    first = (p.x & 1) * R;
    at0 = (size_t)(p.x & ~1) * R + r;
    stride = 2 * R;
  } else if (on && i < t) {
    const int r0 = r / a.rows * a.rows;
    ns = make_span(a, a.lens != nullptr, len, len - t, t, group_of(a, r0), group_of(a, min(r0 + a.rows - 1, R - 1)),
                   a.tile_keys).ns;
  }
  on = ns > 1;   // (a single split has written its row)
  Split o = {-kUnset, 0.f, 0.f, zero4()};
  if (on) o = add_splits<D, false>(a, at0, first, stride, ns, gs, GS, ch);
  if constexpr (GS > 1) {
    part[tid] = o.x;
    psum[0][tid] = o.m;
    psum[1][tid] = o.l;
    psum[2][tid] = o.lx;
    __syncthreads();
    on = on && gs == 0;
    if (on) {
#pragma unroll
      for (int k = 1; k < GS; ++k) {
        const int t = tid + k * CR;
        add_split(o, {psum[0][t], psum[1][t], psum[2][t], part[t]});
      }
    }
  }
  if (on) write_out<E, D>(a, ((size_t)e * a.group + g) * a.tokens + i, ch, o.x, o.m, o.l, o.lx);
}

template <typename E, int D, int RT>
hipError_t launch_rows(const AttendK& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks), th(kAtTh);
  if (a.even) hipLaunchKernelGGL((attend_even_kernel<E, D, RT>), grid, th, 0, s, a);
  else if (a.lens) hipLaunchKernelGGL((attend_kernel<E, D, RT, kTree>), grid, th, 0, s, a);
  else hipLaunchKernelGGL((attend_kernel<E, D, RT, kContiguous>), grid, th, 0, s, a);
  return hipGetLastError();
}

template <typename E, int D>
hipError_t launch_d(const AttendK& a, int rt, hipStream_t s) {
  if constexpr (sizeof(E) == 2) {
    if (rt == 0) return launch_attend_wide(a, D, s);
    if (rt == 2) return launch_rows<E, D, 2>(a, s);
  }
  return launch_rows<E, D, 1>(a, s);
}

template <typename E, int D>
hipError_t launch_ed(const AttendK& a, int rt, hipStream_t s) {
  const hipError_t e = launch_d<E, D>(a, rt, s);
  if (e != hipSuccess || (a.splits == 1 && !a.even) || a.flags) return e;
  // threads that share a value: two, or with many splits a block's all (16 splits of 32
  // units of 128 rows, call 114 -> 110 us with two; 64 splits of 8 units of 8 rows, 100
  // with two, 95 with eight)
  const int64_t rows = (int64_t)a.entries * a.group * a.tokens;
  constexpr int ALL = kAtTh / (D / 4), FEW = 2;
  if (a.splits > kJoinedSplits)
    hipLaunchKernelGGL((combine_kernel<E, D, ALL>), dim3((unsigned)rows), dim3(kAtTh), 0, s, a);
  else
    hipLaunchKernelGGL((combine_kernel<E, D, FEW>), dim3((unsigned)((rows * FEW + ALL - 1) / ALL)),
                       dim3(kAtTh), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Marks of one call's splits: different for every call of a process, and unlike what
// a workspace may hold.
uint64_t next_nonce() {
  static const uint64_t seed = (uint64_t)std::chrono::system_clock::now().time_since_epoch().count();
  static std::atomic<uint64_t> calls{0};
  uint64_t x = seed + 0x9e3779b97f4a7c15ull * ++calls;   // (splitmix64)
  x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;
  x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
  x ^= x >> 31;
  return x != 0 ? x : 1;
}

// Kernel, splits and workspace of a call whose rows see at most `slots` slots
// each, or (ragged) any number up to that.
AttendPlan attend_plan(int entries, int group, int tokens, int d, int dtype, int64_t slots,
                       bool ragged) {
  AttendPlan p;
  const int64_t R = (int64_t)group * tokens;
  const bool bf16 = dtype == GRKV_BF16;
  // two blocks for each compute unit, which hold them at once but for blocks of 32 rows of 128
  // columns (32 units of 20k to 32k keys, 128 rows, 256 / 512 / 1024 blocks: 138 / 116 / 139
  // us; 300 units of 500 to 4000 keys, 64 rows, 512 / 2048: 168 / 180)
  constexpr int64_t target = 512;
  // the wide kernel from 65 rows on, but for calls of few logits, which one launch of small
  // blocks ends first (2 prompts of 564, 11.2 us beside 14.1; 2 units of 120 rows and 1000
  // keys 13.9 and 16.7, 8 units of 128 rows and 2000 keys 20.9 and 19.1)
  if (bf16 && R > 64 && (double)entries * (double)R * (double)slots > kWideLogits) {
    p.rt = 0;
    p.rows = 128;
    p.tile_keys = kWideKeys;
    p.min_tiles = 2;
  } else {
    // rows of a block: 32 read the keys half as often, 16 make twice the blocks and hold
    // twice the waves (32 rows of bf16 over 8000 keys, 16 / 32 rows a block: 24 units 36.3 /
    // 39.0 us, 64 units 68.0 / 63.6, 512 units of 4000 keys 261 / 243).  float32 products
    // take eight times as long: 16 always (512 units of 32 rows over 1000 keys 160 / 185 us)
    p.rt = bf16 && R > 16 && (int64_t)entries * ((R + 31) / 32) >= 64 ? 2 : 1;
    p.rows = 16 * p.rt;
    p.tile_keys = bf16 ? Tile<u16>::KEYS : Tile<float>::KEYS;
    p.min_tiles = 8;
  }
  p.row_groups = (int)((R + p.rows - 1) / p.rows);
  const int64_t tiles = (slots + p.tile_keys - 1) / p.tile_keys;
  const int64_t most = (tiles + p.min_tiles - 1) / p.min_tiles;
  int64_t s = target / ((int64_t)entries * p.row_groups);
  s = s < most ? s : most;
  p.splits = 1;   // a power of two
  if (p.rt == 0) {
    // a tile takes its block 1.35 us, a row's part 0.26 ns to write and read back, the launch
    // that adds them 6 us.  (8 units of 128 rows and 2000 keys, 1 / 2 / 4 / 8 splits: 52 / 34 /
    // 24 / 19 us; 8 prompts of 4 heads and 1000 positions, 1 / 2: 25 / 44; 100 units of 120
    // rows and 300 keys 16 / 28)
    auto cost = [&](int64_t n) {
      return 1.35 * (double)((tiles + n - 1) / n) + (n > 1 ? 6 + 0.26e-3 * (double)(entries * R * n) : 0);
    };
    for (int n = 2; n <= s && n <= 256; n *= 2)
      if (cost(n) < cost(p.splits)) p.splits = n;
  } else {
    while (2 * p.splits <= s && p.splits < 256) p.splits *= 2;
  }
  const int64_t w = (int64_t)entries * p.splits;
  p.grouped = w % 8 == 0 || w >= 64;
  p.blocks = (p.grouped ? (w + 7) / 8 * 8 : w) * p.row_groups;
  p.joined = p.rt > 0 && p.splits > 1 && p.blocks <= kJoinedBlocks &&
             p.splits <= (p.row_groups == 1 ? kJoinedSplits : kJoinedRowSplits);
  p.even = ragged && p.rt > 0 && p.row_groups == 1 && entries <= kEvenEntries &&
           entries * tiles >= kEvenTiles * (int64_t)kEvenBlocks;
  if (p.even) {
    p.joined = 0;
    p.blocks = kEvenBlocks;
  }
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  const size_t rows = p.even ? 2 * (size_t)p.blocks * R : p.splits > 1 ? (size_t)w * R : 0;
  p.opart = 0;
  p.mpart = up(rows * d * sizeof(float));
  p.flags = p.mpart + up(rows * sizeof(float4));
  p.total = p.flags + (p.joined ? up((size_t)w * p.row_groups * sizeof(uint64_t))
                       : p.even ? up((size_t)entries * sizeof(int2)) : 0);
  return p;
}

// What group_of divides by.
void set_group(AttendK& a) {
  a.gshift = 0;
  while ((1ll << a.gshift) < a.group) ++a.gshift;
  a.gmul = (uint32_t)((((1ull << a.gshift) - (uint64_t)a.group) << 32) / (uint64_t)a.group + 1);
}

hipError_t launch_attend(AttendK a, const AttendPlan& p, int d, int dtype, void* workspace,
                         hipStream_t s) {
  a.row_groups = p.row_groups;
  a.splits = p.splits;
  a.min_tiles = p.min_tiles;
  a.grouped = p.grouped;
  a.blocks = p.blocks;
  a.rows = p.rows;
  a.tile_keys = p.tile_keys;
  a.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)d));
  a.opart = (float*)((char*)workspace + p.opart);
  a.mpart = (float4*)((char*)workspace + p.mpart);
  a.flags = p.joined ? (uint64_t*)((char*)workspace + p.flags) : nullptr;
  a.even = p.even ? (int2*)((char*)workspace + p.flags) : nullptr;
  a.nonce = p.joined ? next_nonce() : 0;
  a.split_shift = __builtin_ctz((unsigned)p.splits);
  set_group(a);
  if (dtype == GRKV_BF16) return d == 64 ? launch_ed<u16, 64>(a, p.rt, s) : launch_ed<u16, 128>(a, p.rt, s);
  return d == 64 ? launch_ed<float, 64>(a, p.rt, s) : launch_ed<float, 128>(a, p.rt, s);
}

}  // namespace grkv
