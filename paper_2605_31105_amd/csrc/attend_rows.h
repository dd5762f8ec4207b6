// A few query rows over the tiles of a unit, by a block of four waves: the sums of attend.hip,
// which says how they are formed, for its kernels and for the short ones of a step (chunk.hip).
#pragma once

#include <type_traits>

#include "attend.h"

namespace grkv {

constexpr int kAtWaves = 4;
constexpr int kAtTh = 64 * kAtWaves;

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

template <typename E, int D>
constexpr int kStage = kAtWaves * Tile<E>::KEYS * D * (int)sizeof(E);

// Rows r0 .. r0 + 16 RT - 1 of entry e over the tiles vt0 .. vt1 - 1 of its span, by a block:
// partial rows from `part` on (passed to other blocks of the launch with `shared`) or,
// with kWhole, the outputs.  v0_s and v1_s: two arrays of kStage bytes in LDS (arrays of their
// own, so that the compiler can tell which of them a load into LDS is for).
template <typename E, int D, int RT, Rows KIND>
__device__ __forceinline__ void attend_rows(const AttendK& a, const Span& sn, int e, int r0, int vt0,
                                            int vt1, int64_t part, bool shared, int len, int t,
                                            const int32_t* trow, char* v0_s, char* v1_s) {
  constexpr bool PAGED = KIND != kContiguous, TREE = KIND == kTree;
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
  if (TREE) draft_family(a, e, t, base, lane, &family, &depth);

  // this lane's rows, one per 16-row tile
  Frag qf[RT][DS];
  RowSight sight[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + 16 * rt + l16;
    const int i = group_of(a, r), g = r - i * a.group;
    const bool on = r < R && i < t;
    sight[rt] = row_sight<TREE>(a, base, i, on, family, depth);
    const E* q = (const E*)a.q + row_at<KIND>(a, e, g, i) * D;
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
  // the first slot of 16-row part h of the tile at slot0, its page, and the byte offset of its rows
  // (uniform)
  auto slot16 = [&](int slot0, int h) { return __builtin_amdgcn_readfirstlane(min(slot0 + 16 * h, last)); };
  auto page16 = [&](int slot) -> int {
    if (PAGED) return page_of<KIND>(trow, slot >> a.shift);
    return 0;
  };
  auto rows16 = [&](int slot, int p) -> size_t {
    if (PAGED) {
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
  int ahead[KT];   // pages of the tile to be loaded next (a step's kernel: see wide_rows.h)
  auto next_tile = [&](int vt) { return min(vt + kAtWaves, vt1 - 1); };   // (past the end: the last tile again)
  auto load = [&](int vt, char* vs, Frag (&kf)[KT][DS]) __attribute__((always_inline)) {
    const int slot0 = slot_of(vt);
    size_t rb[KT];
#pragma unroll
    for (int h = 0; h < KT; ++h) {
      const int slot = slot16(slot0, h);
      rb[h] = rows16(slot, KIND == kChunk ? ahead[h] : page16(slot));
      if (KIND == kChunk) ahead[h] = page16(slot16(slot_of(next_tile(vt)), h));
    }
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
    load(next_tile(vt), nxt, kn);
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
        const uint32_t on = sees32<TREE>(sight[rt], slot0, a.n_sink, base, len) >> (4 * gq);
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
#pragma unroll
    for (int h = 0; h < KT; ++h)
      if (KIND == kChunk) ahead[h] = page16(slot16(slot_of(vt), h));
    load(vt, va, ka);
    const bool turns = KIND == kChunk && younger_block();
    for (;;) {
      if (turns) __builtin_amdgcn_s_setprio(1);
      step(vt, va, vc, ka, kc);
      vt += kAtWaves;
      if (vt >= vt1) break;
      if (turns) __builtin_amdgcn_s_setprio(0);
      step(vt, vc, va, kc, ka);
      vt += kAtWaves;
      if (vt >= vt1) break;
    }
  }

  // the waves' parts: references, then rows scaled to the largest, summed over
  // the waves in order.  Every load in flight has to land before its stage is
  // written here.
  if (KIND == kChunk) __builtin_amdgcn_s_setprio(0);
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
    if (TREE) draft_family(a, e, t, base, lane, &family, &depth);   // (not held until here)
    rows_by_key<E, D, KIND>(a, sn, e, part, r0 + wave * (4 * RT), 4 * RT, vt0, vt1, TK, len, t, trow,
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
    if (part != kWhole) {
      put4(a.opart + (part + r) * D + 4 * ch, x, shared);
      if (ch == 0) put4((float*)(a.mpart + part + r), (f32x4){m, l * up, l, 0.f}, shared);
    } else {
      write_out<E, D>(a, row_at<KIND>(a, e, g, i), ch, x, m, l * up, l);
    }
  }
}

}  // namespace grkv
