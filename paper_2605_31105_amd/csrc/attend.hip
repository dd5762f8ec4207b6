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
#include "attend.h"

#include <atomic>
#include <chrono>
#include <type_traits>

namespace grkv {
namespace {

constexpr int kAtWaves = 4;
constexpr int kAtTh = 64 * kAtWaves;
constexpr float kPartUp = 1.f + 0x1p-18f;   // of a weight, before its upper bits are taken away
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

// 16 bytes per lane from memory to LDS, lane after lane from `lds` (uniform), as
// a non-temporal load: values are read once, and pass the caches faster so (over
// caches used in turn: 256 units of 4100 keys 99 -> 89 us, 8 of 128k 103 -> 95, 512 of
// 4250 217 -> 204).  Keys too: 89, 94 and 212 us.
__device__ __forceinline__ void load_lds16(const char* from, char* lds) {
  constexpr int kNonTemporal = 2;
  __builtin_amdgcn_global_load_lds(from, (lds_void*)lds, 16, 0, kNonTemporal);
}

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <typename E>
struct Tile {
  static constexpr int KEYS = sizeof(E) == 2 ? 32 : 16;   // keys of a wave's tile
  static constexpr int KT = KEYS / 16;
};

// Rows r0 .. r0 + 16 RT - 1 of entry e over the tiles vt0 .. vt1 - 1 of its span, by a block:
// partial rows from `part` on (passed to other blocks of the launch with `shared`) or,
// with part < 0, the outputs.
template <typename E, int D, int RT, bool PAGED>
__device__ __forceinline__ void attend_rows(const AttendK& a, const Span& sn, int e, int r0, int vt0,
                                            int vt1, int64_t part, bool shared, int len, int t,
                                            const int32_t* trow) {
  constexpr bool BF = sizeof(E) == 2;
  constexpr int TK = Tile<E>::KEYS, KT = Tile<E>::KT;
  constexpr int RB = D * (int)sizeof(E);          // bytes of a row
  constexpr int CPR = RB / 16;                    // 16-byte chunks of a row
  constexpr int VB = TK * RB;                     // bytes of a wave's V tile
  constexpr int NV = VB / 1024;                   // its load instructions
  constexpr int RPI = 64 / CPR;                   // rows of one of them
  constexpr int DS = BF ? D / 32 : D / 16;        // 16-byte K fragments of a key
  constexpr int DT = D / 16;
  constexpr int CR = D / 4;                       // 4-value chunks of a row
  static_assert(2 * VB == 16 * 2 * D * 4, "two stages hold the partial rows of a wave");
  typedef typename std::conditional<BF, bf16x8, float4>::type Frag;

  __shared__ __attribute__((aligned(16))) char v0_s[kAtWaves * VB];
  __shared__ __attribute__((aligned(16))) char v1_s[kAtWaves * VB];
  __shared__ float m_s[kAtWaves][16 * RT], l_s[kAtWaves][16 * RT];

  // (what follows from it is formed anew for each unit of a block's part, not held over that
  // loop: float32 of 128 columns in 213 registers instead of 254 and spills, 300 units of
  // 500 to 4000 keys 136 -> 129 us)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, gq = lane >> 4;
  const int R = a.group * a.tokens, base = len - t;

  uint64_t family = 0;
  int depth = 0;
  if (PAGED) draft_family(a, e, t, base, lane, &family, &depth);

  // this lane's rows, one per 16-row tile
  Frag qf[RT][DS];
  RowSight sight[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + 16 * rt + l16;
    const int i = group_of(a, r), g = r - i * a.group;
    const bool on = r < R && i < t;
    sight[rt] = row_sight<PAGED>(a, base, i, on, family, depth);
    const E* q = (const E*)a.q + (((size_t)e * a.group + g) * a.tokens + i) * D;
#pragma unroll
    for (int ks = 0; ks < DS; ++ks) {
      if (on) qf[rt][ks] = *reinterpret_cast<const Frag*>(q + (BF ? 32 * ks + 8 * gq : 16 * ks + 4 * gq));
      else qf[rt][ks] = Frag{};
    }
  }

  // lane offsets inside a tile
  uint32_t ko[KT], vo[NV];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) ko[kt] = l16 * RB + gq * 16;
  auto swz = [](int row) {
    return BF ? (D == 128 ? row & 15 : (row >> 1) & 7) : ((row >> 2) & 3) << 2;
  };
#pragma unroll
  for (int it = 0; it < NV; ++it) {
    const int row = it * RPI + lane / CPR;
    vo[it] = ((row & 15) * CPR + ((lane % CPR) ^ swz(row))) * 16;
  }
  const char* kb = (const char*)a.k;
  const char* vb = (const char*)a.v;
  const int last = sn.kend - 1;
  auto slot_of = [&](int vt) { return (vt < sn.at ? vt : vt - sn.at + sn.bt) * TK; };
  // byte offset of the 16 rows around `slot` (uniform)
  auto rows16 = [&](int slot) -> size_t {
    if (PAGED) {
      int p = trow[slot >> a.shift];
      p = (unsigned)p < (unsigned)a.pages ? p : 0;
      return (((size_t)p << a.shift) + ((slot & ((1 << a.shift) - 1)) & ~15)) * RB;
    }
    return ((size_t)e * a.n + (slot & ~15)) * RB;
  };

  f32x4 acc[DT][RT];
  float nref[RT], sum[RT];   // sum: this lane's weights
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    nref[rt] = kUnset;
    sum[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt][rt] = zero4();
  }

  // loads of tile vt: V into the stage `vs`, then K into registers (in that
  // order: the K fragments' arrival says that V has arrived too).  Rows past the
  // last slot read the last one again.
  auto load = [&](int vt, char* vs, Frag (&kf)[KT][DS]) __attribute__((always_inline)) {
    const int slot0 = slot_of(vt);
    size_t rb[KT];
#pragma unroll
    for (int h = 0; h < KT; ++h)
      rb[h] = rows16(__builtin_amdgcn_readfirstlane(min(slot0 + 16 * h, last)));
    const bool whole = slot0 + TK - 1 <= last;
    auto lane_row = [&](int row) { return min(slot0 + row, last) & 15; };
    // the stage's last reads are done before its refill is asked for
    wait_lds();
#pragma unroll
    for (int it = 0; it < NV; ++it) {
      const int h = (it * RPI) / 16;
      uint32_t o = vo[it];
      if (!whole) {
        const int row = it * RPI + lane / CPR;
        o = (lane_row(row) * CPR + ((lane % CPR) ^ swz(row))) * 16;
      }
      load_lds16(vb + rb[h] + o, vs + it * 1024);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      uint32_t o = ko[kt];
      if (!whole) o = lane_row(16 * kt + l16) * RB + gq * 16;
#pragma unroll
      for (int ks = 0; ks < DS; ++ks)
        kf[kt][ks] = *reinterpret_cast<const Frag*>(kb + rb[kt] + o + ks * 64);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  auto step = [&](int vt, char* vs, char* nxt, const Frag (&kf)[KT][DS], Frag (&kn)[KT][DS])
                  __attribute__((always_inline)) {
    load(min(vt + kAtWaves, vt1 - 1), nxt, kn);   // (past the end: the last tile again)
    const int slot0 = slot_of(vt);
    const bool full = slot0 + TK <= sn.lim && (slot0 >= sn.lo || slot0 + TK <= a.n_sink);
    // s[kt][rt][i]: slot slot0 + 16 kt + 4 gq + i of row l16
    f32x4 s[KT][RT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        s[kt][rt] = zero4();
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
          if constexpr (BF) {
            s[kt][rt] = mfma_bf16(kf[kt][ks], qf[rt][ks], s[kt][rt]);
          } else {
            s[kt][rt] = mfma_f32(kf[kt][ks].x, qf[rt][ks].x, s[kt][rt]);
            s[kt][rt] = mfma_f32(kf[kt][ks].y, qf[rt][ks].y, s[kt][rt]);
            s[kt][rt] = mfma_f32(kf[kt][ks].z, qf[rt][ks].z, s[kt][rt]);
            s[kt][rt] = mfma_f32(kf[kt][ks].w, qf[rt][ks].w, s[kt][rt]);
          }
        }
      }
    if (!full) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const uint32_t on = sees32<PAGED>(sight[rt], slot0, a.n_sink, base, len) >> (4 * gq);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((on >> (16 * kt + i) & 1) == 0) s[kt][rt][i] = -__builtin_huge_valf();
      }
    }
    bool moved = false;
    float mx[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mx[rt] = s[0][rt][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[rt] = fmaxf(mx[rt], s[kt][rt][i]);
      moved |= !(fmaf(mx[rt], a.scale_log2, nref[rt]) <= 0.f);
    }
    if (__any(moved)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float m4 = max_over_groups(mx[rt]);
        if (!(fmaf(m4, a.scale_log2, nref[rt]) <= 0.f) && m4 > -__builtin_huge_valf()) {
          const float ref = fmaf(m4, a.scale_log2, kRefAbove);
          const float f = __builtin_amdgcn_exp2f(-nref[rt] - ref);
          nref[rt] = -ref;
          sum[rt] *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt][rt] *= f;
        }
      }
    }
    // the weights; a slot that is not seen has logit -inf and weight 0
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[kt][rt][i] = __builtin_amdgcn_exp2f(fmaf(s[kt][rt][i], a.scale_log2, nref[rt]));
          sum[rt] += s[kt][rt][i];
        }

    // V^T operand of output columns 16 dt ..: bf16 by the transpose read (lane
    // 4e + q of a group supplies row 4 gq + e, columns 4q .. 4q + 3), float32 one
    // value of row 4 gq + i
    const int row_t = 4 * gq + (l16 >> 2);
    const int at_t = row_t * RB + ((((l16 >> 1) & 1) ^ swz(row_t)) << 4) + ((l16 & 1) << 3);
    auto frag = [&](int dt) {
      const char* p0 = vs + (at_t ^ (dt << 5));
      // (the chunk order of rows 16 .. 31 is that of rows 0 .. 15)
      const v4i16 x = ds_read_tr16(p0), y = ds_read_tr16(p0 + 16 * RB);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto elem = [&](int dt, int i) {
      const int row = 4 * gq + i, ch = 4 * dt + (l16 >> 2);
      return *reinterpret_cast<const float*>(vs + (row * CPR + (ch ^ swz(row))) * 16 + 4 * (l16 & 3));
    };
    bf16x8 p[RT], pl[RT];   // the two parts of the weights
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if constexpr (BF) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const uint32_t w0 = __float_as_uint(s[kt][rt][i]), w1 = __float_as_uint(s[kt][rt][i + 1]);
            const bf16x2 h = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(w1, w0, 0x07060302u));
            const f32x2 r = {fmaf(s[kt][rt][i], kPartUp, -__uint_as_float(w0 & 0xffff0000u)),
                             fmaf(s[kt][rt][i + 1], kPartUp, -__uint_as_float(w1 & 0xffff0000u))};
            const bf16x2 l = __builtin_convertvector(r, bf16x2);
            p[rt][4 * kt + i] = h[0];
            p[rt][4 * kt + i + 1] = h[1];
            pl[rt][4 * kt + i] = l[0];
            pl[rt][4 * kt + i + 1] = l[1];
          }
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if constexpr (BF) {
        const bf16x8 vf = frag(dt);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[dt][rt] = mfma_bf16(vf, p[rt], acc[dt][rt]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[dt][rt] = mfma_bf16(vf, pl[rt], acc[dt][rt]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float vf = elem(dt, i);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[dt][rt] = mfma_f32(vf, s[0][rt][i], acc[dt][rt]);
        }
      }
    }
  };
  char* va = v0_s + wave * VB;
  char* vc = v1_s + wave * VB;
  int vt = vt0 + wave;
  if (vt < vt1) {
    Frag ka[KT][DS], kc[KT][DS];
    load(vt, va, ka);
    for (;;) {
      step(vt, va, vc, ka, kc);
      vt += kAtWaves;
      if (vt >= vt1) break;
      step(vt, vc, va, kc, ka);
      vt += kAtWaves;
      if (vt >= vt1) break;
    }
  }

  // the waves' parts: references, then rows scaled to the largest, summed over
  // the waves in order.  Every load in flight has to land before its stage is
  // written here.
  wait_vmcnt<0>();
  bool odd = false, far = false;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 16);
    sum[rt] += __shfl_xor(sum[rt], 32);
    float z = 0.f;   // NaN if a sum of values is not finite
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) z = fmaf(acc[dt][rt][i], 0.f, z);
    odd |= z != z && sum[rt] == sum[rt];
    far |= far_off(sum[rt], nref[rt]);
  }
  if (__syncthreads_or(odd || far) &&
      (__syncthreads_or(far) || odd_values<E, D, PAGED>(a, sn, e, vt0, vt1, TK, sn.lim, sn.lo, trow))) {
    if (PAGED) draft_family(a, e, t, base, lane, &family, &depth);   // (not held until here)
    rows_by_key<E, D, PAGED>(a, sn, e, part, r0 + wave * (4 * RT), 4 * RT, vt0, vt1, TK, len, t, trow,
                             family, depth);
    return;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (gq == 0) {
      m_s[wave][16 * rt + l16] = -nref[rt];
      l_s[wave][16 * rt + l16] = sum[rt];
    }
  }
  __syncthreads();
  char* mine = (wave < 2 ? v0_s : v1_s) + (wave & 1) * 2 * VB;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = 16 * rt + l16;
    float m = m_s[0][row];
#pragma unroll
    for (int w = 1; w < kAtWaves; ++w) m = fmaxf(m, m_s[w][row]);
    const float f = __builtin_amdgcn_exp2f(-nref[rt] - m);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4*>(mine + row * D * 4 + (((4 * dt + gq) ^ l16) << 4)) = acc[dt][rt] * f;
  }
  __syncthreads();
  const float up = BF ? kPartUp : 1.f;   // (what the parts add up to, of a weight)
  for (int c = tid; c < 16 * RT * CR; c += kAtTh) {
    const int row = c / CR, ch = c % CR, r = r0 + row;
    const int i = group_of(a, r), g = r - i * a.group;
    if (r >= R || i >= t) continue;
    float m = m_s[0][row], l = 0.f;
#pragma unroll
    for (int w = 1; w < kAtWaves; ++w) m = fmaxf(m, m_s[w][row]);
    f32x4 x = zero4();
#pragma unroll
    for (int w = 0; w < kAtWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][row] - m);
      l += l_s[w][row] * f;
      x += *reinterpret_cast<const f32x4*>((w < 2 ? v0_s : v1_s) + (w & 1) * 2 * VB + row * D * 4 +
                                           ((ch ^ (row & 15)) << 4));
    }
    if (part >= 0) {
      put4(a.opart + (part + r) * D + 4 * ch, x, shared);
      if (ch == 0) put4((float*)(a.mpart + part + r), (f32x4){m, l * up, l, 0.f}, shared);
    } else {
      const size_t at = ((size_t)e * a.group + g) * a.tokens + i;
      write_out<E, D>(a, at, ch, x, m, l * up, l);
    }
  }
}

template <typename E, int D, int RT, bool PAGED>
__global__ __launch_bounds__(kAtTh, RT == 2 && D == 128 ? 1 : 2) void attend_kernel(AttendK a) {
  int e, rg, sp;
  if (!block_work(a, &e, &rg, &sp)) return;
  const int R = a.group * a.tokens, r0 = rg * 16 * RT;
  int len, t;
  const int32_t* trow;
  entry_shape(a, e, &len, &t, &trow);
  const Span sn = make_span(a, len, len - t, t, group_of(a, r0), group_of(a, min(r0 + 16 * RT - 1, R - 1)),
                            Tile<E>::KEYS);
  const int vt0 = sp * sn.chunk, vt1 = min(sn.nt, vt0 + sn.chunk);
  if (sp > 0 && vt0 >= sn.nt) return;
  attend_rows<E, D, RT, PAGED>(a, sn, e, r0, vt0, vt1, sn.ns > 1 ? ((int64_t)e * a.splits + sp) * R : -1,
                               a.flags != nullptr, len, t, trow);

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
  const Span sn = make_span(a, len, len - t, t, 0, group_of(a, min(16 * RT - 1, R - 1)), Tile<E>::KEYS);
  *tiles = max(sn.nt, 1);
  return sn;
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | lo);
}

// Units of any lengths, one row group each: the tiles of all of them in a row, cut into
// as many equal parts as there are blocks, so that no block waits for a longer one.  A
// part goes over the ends of units; of the rows of a part only the first and the last
// unit's may be partial.  Every block adds up the lengths for itself.
template <typename E, int D, int RT>
__global__ __launch_bounds__(kAtTh, RT == 2 && D == 128 ? 1 : 2) void attend_even_kernel(AttendK a) {
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
    attend_rows<E, D, RT, true>(a, sn, e, 0, vt0, min(vt1, sn.nt), whole ? -1 : slot * R, false, len, t, trow);
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
    ns = make_span(a, len, len - t, t, group_of(a, r0), group_of(a, min(r0 + a.rows - 1, R - 1)), a.tile_keys).ns;
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
  else if (a.lens) hipLaunchKernelGGL((attend_kernel<E, D, RT, true>), grid, th, 0, s, a);
  else hipLaunchKernelGGL((attend_kernel<E, D, RT, false>), grid, th, 0, s, a);
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
static uint64_t next_nonce() {
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
  a.gshift = 0;
  while ((1ll << a.gshift) < a.group) ++a.gshift;
  a.gmul = (uint32_t)((((1ull << a.gshift) - (uint64_t)a.group) << 32) / (uint64_t)a.group + 1);
  if (dtype == GRKV_BF16) return d == 64 ? launch_ed<u16, 64>(a, p.rt, s) : launch_ed<u16, 128>(a, p.rt, s);
  return d == 64 ? launch_ed<float, 64>(a, p.rt, s) : launch_ed<float, 128>(a, p.rt, s);
}

}  // namespace grkv
