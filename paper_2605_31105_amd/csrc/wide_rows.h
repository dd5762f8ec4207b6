// Many query rows (bf16) over the tiles of a unit, by a block of four waves: the sums of
// attend_wide.hip, which says how they are formed, for its kernel and for the chunks of a
// step (chunk.hip).
#pragma once

#include "attend.h"

namespace grkv {

constexpr int kWWaves = 4;
constexpr int kWTh = 64 * kWWaves;

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// The barrier of the ring: this wave's loads but the last N have landed, and its
// reads are done.
template <int N>
__device__ __forceinline__ void ring_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ bf16x8 read_tr(const char* p, int rows8) {
  const v4i16 x = ds_read_tr16(p), y = ds_read_tr16(p + rows8);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Where a block's rows go: partial rows from `row` on, or the outputs.
struct Part {
  bool partial;
  int64_t row;
};

template <int D>
constexpr int kRing = 2 * kWideKeys * 2 * D;   // bytes of either ring

// Rows r0 .. r0 + 127 of entry e over the tiles vt0 .. vt1 - 1 of its span, by a block: partial
// rows from part_of() on or (kWhole) the outputs.  kring and vring: two tiles of keys and two of
// values in LDS, 1 KB aligned.  TWO: 64 rows at most, whose weights enter their product in two bf16
// parts, as in attend.hip.  Waves w and w + 2 hold the same 32 rows and take half of a tile's keys each
// (two waves would have none), and their sums are added at the end.
template <int D, Rows KIND, bool TWO = false, typename F>
__device__ __forceinline__ void wide_rows(const AttendK& a, const Span& sn, int e, int r0, int vt0, int vt1,
                                          F part_of, int len, int t, const int32_t* trow, char* kring,
                                          char* vring) {
  constexpr bool PAGED = KIND != kContiguous, TREE = KIND == kTree;
  constexpr int TK = kWideKeys;
  constexpr int NK = TWO ? 1 : TK / 32;   // 32-key parts of a wave's step
  constexpr int RB = 2 * D;            // bytes of a row
  constexpr int CPR = RB / 16;         // chunks of a row
  constexpr int KB = TK * RB;          // bytes of a K (or V) tile
  constexpr int NI = 16 * RB / 1024;   // load instructions per wave and tensor: 16 rows
  constexpr int RPI = 64 / CPR;        // rows of one
  constexpr int KS = D / 16, DM = D / 32;
  static_assert(TK == 16 * kWWaves, "a wave brings 16 rows of a tile");
  static_assert(kWWaves * 32 * D * 4 == 2 * kRing<D>, "the waves' outputs fit the ring");
  static_assert(!TWO || (KIND == kChunk && kWWaves == 4), "the jobs of a step");

  int tid = threadIdx.x;
  if (KIND == kChunk) asm volatile("" : "+v"(tid));   // (what follows from it is not held over jobs)
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int R = a.group * a.tokens, base = len - t;

  uint64_t family = 0;
  int depth = 0;
  if (TREE) draft_family(a, e, t, base, lane, &family, &depth);
  const int w0 = r0 + 32 * (TWO ? wave & 1 : wave);   // this wave's first row
  const int key0 = TWO ? 32 * (wave >> 1) : 0;           // its first key of a tile
  bf16x8 qf[KS];
  RowSight sight;
  {
    const int r = w0 + l32;
    const int i = group_of(a, r), g = r - i * a.group;
    const bool on = r < R && i < t;
    sight = row_sight<TREE>(a, base, i, on, family, depth);
    const u16* q = (const u16*)a.q + row_at<KIND>(a, e, g, i) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (on) qf[ks] = *reinterpret_cast<const bf16x8*>(q + 16 * ks + 8 * h);
      else qf[ks] = bf16x8{};
    }
  }
  // slots that every row of the wave sees: before lim and from lo on, or sinks
  int lim = sn.lim, lo = sn.lo;
  if (!TREE) {
    lim = base + group_of(a, min(w0, R - 1)) + 1;
    lo = a.window > 0 ? base + group_of(a, min(w0 + 31, R - 1)) + 1 - a.window : 0;
  }

  // ---- loads: this wave brings rows 16 wave .. + 15 of every tile
  auto swz_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto swz_v = [](int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; };
  // (lane's byte in the first kilobyte; the rows of the next ones are 1 KB on, where K's chunks
  // are also permuted by 4)
  const int row0 = lane / CPR, ch0 = lane % CPR;
  const uint32_t ko = (row0 * CPR + (ch0 ^ swz_k(row0))) * 16, vo = (row0 * CPR + (ch0 ^ swz_v(row0))) * 16;
  static_assert(RPI == 4 || RPI == 8, "rows of a kilobyte");
  const int last = sn.kend - 1;
  const uint32_t kr0 = (uint32_t)(uintptr_t)(lds_void*)kring;
  const uint32_t vr0 = KIND == kChunk ? (uint32_t)(uintptr_t)(lds_void*)vring : kr0 + 2 * KB;
  auto slot_of = [&](int vt) { return (vt < sn.at ? vt : vt - sn.at + sn.bt) * TK; };
  // this wave's first slot of tile vt, its page, and its row
  auto wave_slot = [&](int vt) { return __builtin_amdgcn_readfirstlane(min(slot_of(vt) + 16 * wave, last)); };
  auto page_at = [&](int vt) -> int {
    if (PAGED) return page_of<KIND>(trow, wave_slot(vt) >> a.shift);
    return 0;
  };
  auto row_in = [&](int vt, int p) -> size_t {
    const int at = wave_slot(vt);
    if (!PAGED) return (size_t)e * a.n + (at & ~15);
    p = (unsigned)p < (unsigned)a.pages ? p : 0;
    return ((size_t)p << a.shift) + ((at & ((1 << a.shift) - 1)) & ~15);
  };
  // this wave's rows of tile vt in page p, of K or V (o: its lane offset; step: how the next
  // kilobyte's differs)
  auto load = [&](const void* from, int vt, int p, uint32_t to, uint32_t o, int step, bool once)
                  __attribute__((always_inline)) {
    const int s16 = slot_of(vt) + 16 * wave;
    const char* src = (const char*)from + row_in(vt, p) * RB;
    const uint32_t dst = __builtin_amdgcn_readfirstlane(to + wave * 16 * RB);
    auto bring = [&](const char* at, uint32_t f, int it) __attribute__((always_inline)) {
      if (once) ring_load<true>(at, f, dst + it * 1024);
      else ring_load(at, f, dst + it * 1024);
    };
    if (s16 + 15 <= last) {
#pragma unroll
      for (int it = 0; it < NI; ++it) bring(src + it * 1024, o ^ (it * step), it);
    } else {   // rows past the last slot: the last one again
      int l = lane;
      asm volatile("" : "+v"(l));   // (formed here, not held over the loop)
#pragma unroll
      for (int it = 0; it < NI; ++it)
        bring(src, (min(s16 + it * RPI + l / CPR, last) & 15) * RB + ((o ^ (it * step)) & (RB - 1)), it);
    }
  };

  // ---- operand reads.  K: lane's key l32, chunk 2 ks + h.  V: the transpose read's
  // lane 4 e + q of a 16-lane group supplies key 4 h + e (+ 8 in the second half),
  // columns 32 dm + 16 (lane / 16 % 2) + 4 q ..
  const int e4 = (lane >> 2) & 3, q4 = lane & 3;
  const int ka = l32 * RB + ((h ^ swz_k(l32)) << 4);
  const int va = (4 * h + e4) * RB +
                 (((2 * ((lane >> 4) & 1) + (q4 >> 1)) ^ swz_v(4 * h + e4)) << 4) + (q4 & 1) * 8;
  auto read_k = [&](const char* tile, bf16x8 (&kf)[KS]) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      kf[ks] = *reinterpret_cast<const bf16x8*>(tile + (ka ^ (ks << 5)));
  };
  auto read_v = [&](const char* tile, bf16x8 (&vf)[2][DM]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int dm = 0; dm < DM; ++dm)
        vf[s][dm] = read_tr(tile + 16 * s * RB + (va ^ (dm << 6)), 8 * RB);
  };

  f32x16 acc[DM], s0[NK];
  float nref = kUnset;          // minus the reference
  float sum = 0.f, rsum = 0.f;  // weights' sums before and after their rounding (this lane's keys)
#pragma unroll
  for (int dm = 0; dm < DM; ++dm) acc[dm] = f32x16{};

  auto logits = [&](const char* kt, f32x16 (&x)[NK]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      bf16x8 kf[KS];
      read_k(kt + (key0 + n * 32) * RB, kf);
      x[n] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x[n] = mfma32(kf[ks], qf[ks], x[n]);
    }
  };
  // One step: the 32 NK keys at key0 of the tile at `slot`, whose logits are in st and whose V rows are
  // at vt; kt: K rows of the next step.
  auto step = [&](int slot, const char* kt, const char* vt, f32x16 (&st)[NK], f32x16 (&nx)[NK])
                  __attribute__((always_inline)) {
    const int slot0 = slot + key0;
    const bool full = slot0 + 32 * NK <= lim && (slot0 >= lo || slot0 + 32 * NK <= a.n_sink);
    if (!full) {
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        const uint32_t on = sees32<TREE>(sight, slot0 + 32 * n, a.n_sink, base, len) >> (4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((on >> (8 * (r / 4) + r % 4) & 1) == 0) st[n][r] = -__builtin_huge_valf();
      }
    }
    logits(kt, nx);
    bf16x8 p[NK][2], rest[TWO ? NK : 1][2];
    float s1, s2;   // this step's sums
    auto weights = [&]() __attribute__((always_inline)) {
      s1 = s2 = 0.f;
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int c = 0; c < 8; c += 2) {
            const float x0 = __builtin_amdgcn_exp2f(fmaf(st[n][8 * s + c], a.scale_log2, nref));
            const float x1 = __builtin_amdgcn_exp2f(fmaf(st[n][8 * s + c + 1], a.scale_log2, nref));
            s1 += x0;
            s1 += x1;
            bf16x2 w;
            if constexpr (TWO) {
              const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
              w = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(u1, u0, 0x07060302u));
              const bf16x2 l = __builtin_convertvector((f32x2){fmaf(x0, kPartUp, -__uint_as_float(u0 & 0xffff0000u)),
                                                               fmaf(x1, kPartUp, -__uint_as_float(u1 & 0xffff0000u))},
                                                       bf16x2);
              rest[n][s][c] = l[0];
              rest[n][s][c + 1] = l[1];
            } else {
              w = __builtin_convertvector((f32x2){x0, x1}, bf16x2);
              s2 = __builtin_amdgcn_fdot2_f32_bf16(w, __builtin_bit_cast(bf16x2, kOnes), s2, false);
            }
            p[n][s][c] = w[0];
            p[n][s][c + 1] = w[1];
          }
    };
    weights();
    bool moved = !(s1 <= kMoveSum);
    if (__any(moved)) {   // (also the first logits that a row sees)
      moved |= __shfl_xor((int)moved, 32) != 0;
      float mx = st[0][0];
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[n][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (moved && mx > -__builtin_huge_valf()) {
        const float ref = mx * a.scale_log2;
        const float f = __builtin_amdgcn_exp2f(-nref - ref);
        nref = -ref;
        sum *= f;
        rsum *= f;
#pragma unroll
        for (int dm = 0; dm < DM; ++dm) acc[dm] *= f;
      }
      weights();
    }
    sum += s1;
    rsum += s2;
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      bf16x8 vf[2][DM];
      read_v(vt + (key0 + n * 32) * RB, vf);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int dm = 0; dm < DM; ++dm) {
          acc[dm] = mfma32(vf[s][dm], p[n][s], acc[dm]);
          if constexpr (TWO) acc[dm] = mfma32(vf[s][dm], rest[n][s], acc[dm]);
        }
    }
    // products of the step, operands read ahead.  (Left to itself the compiler reads two ahead in
    // a step's kernel, and the products wait for LDS: 4 chunks of 2048 over 4k to 14k 1620 -> 1500
    // us; three to eight ahead are equal.  A 16k prompt over 8 units 2274 -> 2248; trees are as fast
    // without.)
    constexpr int ALL = NK * 2 * DM, AHEAD = 4, EACH = TWO ? 2 : 1;
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
    for (int k = 0; k < ALL - AHEAD; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, EACH * AHEAD, 0);
  };

  if (vt0 < vt1) {
    // values that no other row group reads are read once (32 units of 20k to 32k keys,
    // over caches used in turn, 116 -> 114 us; keys too, 114)
    const bool once = TREE && a.row_groups == 1;
    // tile i is in half i & 1 of either ring
    auto tile = [&](int i) { return min(vt0 + i, vt1 - 1); };
    auto load_k = [&](int i, int p) { load(a.k, tile(i), p, kr0 + (i & 1) * KB, ko, 64, false); };
    auto load_v = [&](int i, int p) { load(a.v, tile(i), p, vr0 + (i & 1) * KB, vo, 0, once); };
    const int p0 = page_at(tile(0));
    // A step's pages are looked up a step before their keys are asked for, and values take those
    // of the keys, so that no step waits for the table (4 chunks of 2048 over 4k to 14k 1564 ->
    // 1524 us).
    int pv = page_at(tile(1)), pk = 0;
    load_k(0, p0);
    load_k(1, pv);
    load_v(0, p0);
    if (KIND == kChunk) pk = page_at(tile(2));
    ring_barrier<2 * NI>();
    logits(kring, s0);
    if (KIND == kChunk) {
      f32x16 s1[NK];
      const bool turns = younger_block();
      // Two steps to a turn, so that logits are formed where the step after reads them
      // (4 chunks of 2048 over 4k to 14k 1405 -> 1330 us).
      auto turn = [&](int i, int odd, f32x16 (&st)[NK], f32x16 (&nx)[NK]) __attribute__((always_inline)) {
        // K of tile i + 1 and V of tile i are here, and every wave is done with K of
        // tile i and V of tile i - 1
        ring_barrier<0>();
        if (turns) odd ? __builtin_amdgcn_s_setprio(1) : __builtin_amdgcn_s_setprio(0);
        load(a.k, tile(i + 2), pk, kr0 + odd * KB, ko, 64, false);
        load(a.v, tile(i + 1), pv, vr0 + (1 - odd) * KB, vo, 0, false);
        pv = pk;
        pk = page_at(tile(i + 3));
        step(slot_of(vt0 + i), kring + (1 - odd) * KB, vring + odd * KB, st, nx);
      };
      for (int i = 0;;) {
        turn(i, 0, s0, s1);
        if (++i >= vt1 - vt0) break;
        turn(i, 1, s1, s0);
        if (++i >= vt1 - vt0) break;
      }
    } else {
      for (int i = 0; i < vt1 - vt0; ++i) {
        ring_barrier<0>();
        load_k(i + 2, page_at(tile(i + 2)));
        load_v(i + 1, page_at(tile(i + 1)));
        f32x16 nx[NK];
        step(slot_of(vt0 + i), kring + ((i + 1) & 1) * KB, vring + (i & 1) * KB, s0, nx);
#pragma unroll
        for (int n = 0; n < NK; ++n) s0[n] = nx[n];
      }
    }
  }
  if (KIND == kChunk) __builtin_amdgcn_s_setprio(0);
  ring_barrier<0>();   // (the rings are the output's buffer now)
  sum += __shfl_xor(sum, 32);
  rsum += __shfl_xor(rsum, 32);
  float odd = 0.f;   // NaN if a sum of values is not finite
#pragma unroll
  for (int dm = 0; dm < DM; ++dm)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(acc[dm][r], 0.f, odd);
  const Part to = part_of();
  const bool far = far_off(sum, nref);
  if constexpr (TWO) {
    __shared__ float m_s[2][64], l_s[2][64];   // references and sums of the rows over either half of the keys
    if (__syncthreads_or(far || (odd != odd && sum == sum)) &&
        (__syncthreads_or(far) || odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, sn.lim, sn.lo, trow) ||
         !odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, 0, sn.lo, trow))) {
      rows_by_key<u16, D, KIND>(a, sn, e, to.partial ? to.row : kWhole, r0 + 16 * wave, 16, vt0, vt1, TK, len, t, trow,
                                family, depth);
      return;
    }
    // the halves' rows, scaled to the larger reference, through the waves' parts of the rings (lane's
    // four columns 32 dm + 8 c + 4 h of row l32, chunks permuted by row), added where they are read
    constexpr int CR = D / 4;
    const int my = 32 * (wave & 1) + l32;
    if (h == 0) {
      m_s[wave >> 1][my] = -nref;
      l_s[wave >> 1][my] = sum;
    }
    __syncthreads();
    // (of a part: weights of 1 at most, so that parts may be added)
    const float f = __builtin_amdgcn_exp2f(-nref - fmaxf(m_s[0][my], m_s[1][my])) * (to.partial ? 1.f / kMoveSum : 1.f);
    char* mine = (wave < 2 ? kring : vring) + (wave & 1) * KB;
#pragma unroll
    for (int dm = 0; dm < DM; ++dm)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<f32x4*>(mine + (l32 * CR + ((8 * dm + 2 * c + h) ^ (l32 & 15))) * 16) =
            (f32x4){acc[dm][4 * c], acc[dm][4 * c + 1], acc[dm][4 * c + 2], acc[dm][4 * c + 3]} * f;
    __syncthreads();
#pragma unroll 4
    for (int k = tid; k < 64 * CR; k += kWTh) {
      const int row = k / CR, ch = k % CR, r = r0 + row, i = group_of(a, r);
      if (r >= R || i >= t) continue;
      const int at = (row >> 5) * KB + ((row & 31) * CR + (ch ^ (row & 15))) * 16;
      const f32x4 x = *reinterpret_cast<const f32x4*>(kring + at) + *reinterpret_cast<const f32x4*>(vring + at);
      const float m = fmaxf(m_s[0][row], m_s[1][row]);
      const float lx = l_s[0][row] * __builtin_amdgcn_exp2f(m_s[0][row] - m) + l_s[1][row] * __builtin_amdgcn_exp2f(m_s[1][row] - m);
      if (to.partial) {
        const float l = lx * (1.f / kMoveSum);
        *reinterpret_cast<f32x4*>(a.opart + (to.row + r) * D + 4 * ch) = x;
        if (ch == 0) a.mpart[to.row + r] = make_float4(m + kMoveLog, l * kPartUp, l, 0.f);
      } else {
        write_out<u16, D>(a, row_at<KIND>(a, e, r - i * a.group, i), ch, x, m, lx * kPartUp, lx);
      }
    }
    return;
  }
  if (__any(far || (odd != odd && sum == sum)) &&
      (__any(far) || odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, lim, lo, trow) ||
       !odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, 0, lo, trow))) {
    if (TREE) draft_family(a, e, t, base, lane, &family, &depth);   // (not held until here)
    rows_by_key<u16, D, KIND>(a, sn, e, to.partial ? to.row : kWhole, w0, 32, vt0, vt1, TK, len, t, trow, family, depth);
    return;
  }
  // a wave's rows through its part of the ring (lane's four columns 32 dm + 8 c + 4 h of
  // row l32, chunks permuted by row), so that they leave whole
  const int my = w0 + l32, mi = group_of(a, my);
  char* out = KIND == kChunk ? (wave < 2 ? kring : vring) + (wave & 1) * KB : kring + wave * KB;
  if (to.partial) {
    constexpr int CR = D / 4;
    const float fit = 1.f / kMoveSum;   // (weights of 1 at most, so that parts may be added)
#pragma unroll
    for (int dm = 0; dm < DM; ++dm)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<f32x4*>(out + (l32 * CR + ((8 * dm + 2 * c + h) ^ (l32 & 15))) * 16) =
            (f32x4){acc[dm][4 * c], acc[dm][4 * c + 1], acc[dm][4 * c + 2], acc[dm][4 * c + 3]} * fit;
    if (h == 0 && my < R && mi < t)
      a.mpart[to.row + my] = make_float4(kMoveLog - nref, rsum * fit, sum * fit, 0.f);
#pragma unroll 4
    for (int k = lane; k < 32 * CR; k += 64) {
      const int row = k / CR, ch = k % CR, r = w0 + row;
      if (r < R && group_of(a, r) < t)
        *reinterpret_cast<f32x4*>(a.opart + (to.row + r) * D + 4 * ch) =
            *reinterpret_cast<const f32x4*>(out + (row * CR + (ch ^ (row & 15))) * 16);
    }
    return;
  }
  const float inv = rsum == 0.f ? 0.f : 1.f / rsum;
#pragma unroll
  for (int dm = 0; dm < DM; ++dm)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint2 w;
      w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(
          (f32x2){acc[dm][4 * c] * inv, acc[dm][4 * c + 1] * inv}, bf16x2));
      w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(
          (f32x2){acc[dm][4 * c + 2] * inv, acc[dm][4 * c + 3] * inv}, bf16x2));
      *reinterpret_cast<uint2*>(out + (l32 * CPR + ((4 * dm + c) ^ (l32 & (CPR - 1)))) * 16 + 8 * h) = w;
    }
  auto place = [&](int r, int i) { return row_at<KIND>(a, e, r - i * a.group, i); };
  if (h == 0 && a.lse && my < R && mi < t)
    a.lse[place(my, mi)] = sum == 0.f ? -__builtin_huge_valf() : (__log2f(sum) - nref) * kLn2;
#pragma unroll
  for (int k = lane; k < 32 * CPR; k += 64) {
    const int row = k / CPR, ch = k % CPR, r = w0 + row, i = group_of(a, r);
    if (r < R && i < t)
      *reinterpret_cast<uint4*>((u16*)a.o + place(r, i) * D + 8 * ch) =
          *reinterpret_cast<const uint4*>(out + (row * CPR + (ch ^ (row & (CPR - 1)))) * 16);
  }
}

}  // namespace grkv
