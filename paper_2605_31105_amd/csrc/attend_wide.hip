// Attention of many query rows over the keys of a unit (bf16): prompts and chunks
// of them with a window and sinks, trees of drafted tokens with more than 64 rows.
//
// The sums are those of attend.hip; here they are bound by the MFMAs, so a wave
// holds RT tiles of 32 rows (RT = 2: 64 rows, 256 per block) and the four waves
// of a block share tiles of 64 keys in LDS:
//  * K and V go from memory to a ring of four LDS stages (global_load_lds), two
//    tiles ahead, one barrier per tile.  16-byte chunks are permuted by row so
//    that neither the K operand reads nor the V transpose reads conflict.
//  * 32x32x16 MFMAs: S^T = K Q^T leaves a query row in each lane column, where
//    P^T already is the B operand of O^T = V^T P^T.  A fragment read from LDS
//    feeds RT products: with 64 rows a wave the LDS is read at half the rate that
//    the MFMAs could take, with 32 at the whole.
//  * One wave per SIMD, so the products have to run beside the exponentials of the
//    same wave: while the weights of 32 keys of a row tile are formed, the logits
//    of the next 32 keys and the P.V of the row tile before are issued.
//  * The reference of a row is a whole number (base 2) and moves only when a logit
//    passes it by 2^40; the weights in flight are then rescaled exactly.
//  * P is rounded to bf16 and o divided by the sum of the rounded weights; lse is
//    of the weights before.
#include "attend.h"

namespace grkv {
namespace {

constexpr int kWTh = 256;
constexpr int kWStages = 4;

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

// 16 bytes per lane from base + voff to LDS offset lds (uniform), lane after
// lane.  In assembly so that the compiler does not wait for these loads at every
// LDS read; ring_barrier does where it matters.
__device__ __forceinline__ void ring_load(const char* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds)
               : "memory", "m0");
}

__device__ __forceinline__ bf16x8 read_tr(const char* p, int rows8) {
  const v4i16 x = ds_read_tr16(p), y = ds_read_tr16(p + rows8);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int D, int RT, bool PAGED>
__global__ __launch_bounds__(kWTh, 1) void wide_kernel(AttendK a) {
  constexpr int TK = kWideKeys, NS = kWStages;
  constexpr int RB = 2 * D;            // bytes of a row
  constexpr int CPR = RB / 16;         // chunks of a row
  constexpr int KB = TK * RB;          // bytes of a K (or V) tile
  constexpr int SB = 2 * KB;           // of a stage
  constexpr int NI = KB / 4096;        // load instructions per wave and tensor
  constexpr int RPI = 64 / CPR;        // rows of one
  constexpr int KS = D / 16, DM = D / 32;
  constexpr int WR = 32 * RT;          // rows of a wave
  __shared__ __attribute__((aligned(1024))) char ring[NS * SB];

  int e, rg, sp;
  if (!block_work(a, &e, &rg, &sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int R = a.group * a.tokens, r0 = rg * a.rows;
  int len, t;
  const int32_t* trow;
  entry_shape(a, e, &len, &t, &trow);
  const int base = len - t;
  const Span sn = make_span(a, len, base, t, r0 / a.group, min(r0 + a.rows - 1, R - 1) / a.group, TK);
  const int vt0 = sp * sn.chunk, vt1 = min(sn.nt, vt0 + sn.chunk);
  if (sp > 0 && vt0 >= sn.nt) return;

  uint64_t family = 0;
  int depth = 0;
  if (PAGED) draft_family(a, e, t, base, lane, &family, &depth);
  const int w0 = r0 + wave * WR;   // this wave's first row
  bf16x8 qf[RT][KS];
  RowSight sight[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = w0 + 32 * rt + l32;
    const int i = r / a.group, g = r - i * a.group;
    const bool on = r < R && i < t;
    sight[rt] = row_sight<PAGED>(a, base, i, on, family, depth);
    const u16* q = (const u16*)a.q + (((size_t)e * a.group + g) * a.tokens + i) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (on) qf[rt][ks] = *reinterpret_cast<const bf16x8*>(q + 16 * ks + 8 * h);
      else qf[rt][ks] = bf16x8{};
    }
  }
  // slots that every row of the wave sees: before lim and from lo on, or sinks
  int lim = sn.lim, lo = sn.lo;
  if (!PAGED) {
    lim = base + min(w0, R - 1) / a.group + 1;
    lo = a.window > 0 ? base + min(w0 + WR - 1, R - 1) / a.group + 1 - a.window : 0;
  }

  // ---- loads: this wave brings rows 16 wave .. + 15 of every tile
  auto swz_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto swz_v = [](int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; };
  uint32_t ko[NI], vo[NI];
#pragma unroll
  for (int it = 0; it < NI; ++it) {
    const int row = it * RPI + lane / CPR, ch = lane % CPR;
    ko[it] = (row * CPR + (ch ^ swz_k(row))) * 16;
    vo[it] = (row * CPR + (ch ^ swz_v(row))) * 16;
  }
  const int last = sn.kend - 1;
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void*)ring;
  auto slot_of = [&](int vt) { return (vt < sn.at ? vt : vt - sn.at + sn.bt) * TK; };
  auto load = [&](int vt, int stage) {
    const int s16 = slot_of(vt) + 16 * wave;
    const int at = __builtin_amdgcn_readfirstlane(min(s16, last));
    size_t row;
    if (PAGED) {
      int p = trow[at >> a.shift];
      p = (unsigned)p < (unsigned)a.pages ? p : 0;
      row = ((size_t)p << a.shift) + ((at & ((1 << a.shift) - 1)) & ~15);
    } else {
      row = (size_t)e * a.n + (at & ~15);
    }
    const char* kb = (const char*)a.k + row * RB;
    const char* vb = (const char*)a.v + row * RB;
    const uint32_t to = __builtin_amdgcn_readfirstlane(ring0 + stage * SB + wave * 16 * RB);
    if (s16 + 15 <= last) {
#pragma unroll
      for (int it = 0; it < NI; ++it) {
        ring_load(kb, ko[it], to + it * 1024);
        ring_load(vb, vo[it], to + KB + it * 1024);
      }
    } else {   // rows past the last slot: the last one again
#pragma unroll
      for (int it = 0; it < NI; ++it) {
        const int row_in = it * RPI + lane / CPR, ch = lane % CPR;
        const int from = (min(s16 + row_in, last) & 15) * CPR;
        ring_load(kb, (from + (ch ^ swz_k(row_in))) * 16, to + it * 1024);
        ring_load(vb, (from + (ch ^ swz_v(row_in))) * 16, to + KB + it * 1024);
      }
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

  f32x16 acc[RT][DM], st[RT];
  float nref[RT], sum[RT], rsum[RT];   // minus the reference; the weights' sums before and
                                       // after their rounding (this lane's keys)
  bf16x8 pp[2];                        // weights of the last row tile, not yet multiplied
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    nref[rt] = kUnset;
    sum[rt] = rsum[rt] = 0.f;
#pragma unroll
    for (int dm = 0; dm < DM; ++dm) acc[rt][dm] = f32x16{};
  }
  pp[0] = pp[1] = bf16x8{};
  bool odd = false;   // a value that is not finite in a step that is not seen whole

  // One step: 32 keys at slot0, whose logits are in st.  kt: the next 32 keys' K
  // tile rows; vt: these keys' V rows; vp: the fragments that pp waits for.
  auto step = [&](int slot0, const char* kt, const char* vt, bf16x8 (&vp)[2][DM],
                  bf16x8 (&vf)[2][DM]) __attribute__((always_inline)) {
    const bool full = slot0 + 32 <= lim && (slot0 >= lo || slot0 + 32 <= a.n_sink);
    if (!full) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!sees<PAGED>(sight[rt], slot0 + 8 * (r / 4) + 4 * h + r % 4, a.n_sink, base, len))
            st[rt][r] = -__builtin_huge_valf();
    }
    float mx[RT];
    bool moved = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mx[rt] = st[rt][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx[rt] = fmaxf(mx[rt], st[rt][r]);
      moved |= !(fmaf(mx[rt], a.scale_log2, nref[rt]) <= kMoveAt);
    }
    if (__any(moved)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float m2 = fmaxf(mx[rt], __shfl_xor(mx[rt], 32));
        if (!(fmaf(m2, a.scale_log2, nref[rt]) <= kMoveAt) && m2 > -__builtin_huge_valf()) {
          const float ref = ceilf(m2 * a.scale_log2);
          const float f = __builtin_amdgcn_exp2f(-nref[rt] - ref);
          nref[rt] = -ref;
          sum[rt] *= f;
          rsum[rt] *= f;
#pragma unroll
          for (int dm = 0; dm < DM; ++dm) acc[rt][dm] *= f;
          if (rt == RT - 1) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int c = 0; c < 8; ++c) pp[s][c] = (__bf16)((float)pp[s][c] * f);
          }
        }
      }
    }
    auto logits = [&](const bf16x8 (&kf)[KS], int rt) __attribute__((always_inline)) {
      f32x16 x = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x = mfma32(kf[ks], qf[rt][ks], x);
      return x;
    };
    // weights of a row tile, in place, and their sums
    auto weights = [&](int rt, f32x16& x, bf16x8 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale_log2, nref[rt]));
        sum[rt] += x[r];
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          const bf16x2 w = __builtin_convertvector((f32x2){x[8 * s + c], x[8 * s + c + 1]}, bf16x2);
          p[s][c] = w[0];
          p[s][c + 1] = w[1];
          rsum[rt] = __builtin_amdgcn_fdot2_f32_bf16(w, __builtin_bit_cast(bf16x2, kOnes), rsum[rt], false);
        }
    };
    if (!full) {
      read_v(vt, vf);   // (values that are not finite?)
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int dm = 0; dm < DM; ++dm) {
          const uint4 w = __builtin_bit_cast(uint4, vf[s][dm]);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int c = 0; c < 4; ++c)
            odd |= (u[c] & 0x7f80u) == 0x7f80u || (u[c] & 0x7f800000u) == 0x7f800000u;
        }
    }
    bf16x8 kf[KS];
    read_k(kt, kf);
    read_v(vt, vf);
    f32x16 sn_[RT];
    bf16x8 p[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      weights(rt, st[rt], p[rt]);
      sn_[rt] = logits(kf, rt);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int dm = 0; dm < DM; ++dm) {
          if (rt == 0) acc[RT - 1][dm] = mfma32(vp[s][dm], pp[s], acc[RT - 1][dm]);
          else acc[rt - 1][dm] = mfma32(vf[s][dm], p[rt - 1][s], acc[rt - 1][dm]);
        }
    }
    pp[0] = p[RT - 1][0];
    pp[1] = p[RT - 1][1];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) st[rt] = sn_[rt];
  };

  if (vt0 < vt1) {
    auto tile = [&](int i) { return min(vt0 + i, vt1 - 1); };
    load(tile(0), 0);
    load(tile(1), 1);
    load(tile(2), 2);
    ring_barrier<4 * NI>();
    bf16x8 va_[2][DM], vb_[2][DM];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int dm = 0; dm < DM; ++dm) va_[s][dm] = vb_[s][dm] = bf16x8{};
    {
      bf16x8 kf[KS];
      read_k(ring, kf);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        st[rt] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) st[rt] = mfma32(kf[ks], qf[rt][ks], st[rt]);
      }
    }
    for (int i = 0; i < vt1 - vt0; ++i) {
      const char* cur = ring + (i & (NS - 1)) * SB;
      const char* nxt = ring + ((i + 1) & (NS - 1)) * SB;
      const int slot0 = slot_of(vt0 + i);
      step(slot0, cur + 32 * RB, cur + KB, vb_, va_);
      // tile i + 1 is here, and every wave is done with tile i - 1
      ring_barrier<2 * NI>();
      load(tile(i + 3), (i + 3) & (NS - 1));
      step(slot0 + 32, nxt, cur + KB + 32 * RB, va_, vb_);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int dm = 0; dm < DM; ++dm)
        acc[RT - 1][dm] = mfma32(vb_[s][dm], pp[s], acc[RT - 1][dm]);
  }
  ring_barrier<0>();   // (the ring is the output's buffer now)
  if (__any(odd)) {
    rows_by_key<u16, D, PAGED>(a, sn, e, sp, w0, WR, vt0, vt1, TK, len, t, trow, family, depth);
    return;
  }

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 32);
    rsum[rt] += __shfl_xor(rsum[rt], 32);
  }
  // a wave's rows through its own part of the ring: lane's four columns 32 dm +
  // 8 c + 4 h of row l32, chunks permuted by row
  char* out = ring + wave * (NS * SB / 4);
  if (sn.ns > 1) {
    constexpr int CR = D / 4;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int dm = 0; dm < DM; ++dm)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int ch = 8 * dm + 2 * c + h;
          *reinterpret_cast<f32x4*>(out + (l32 * CR + (ch ^ (l32 & 15))) * 16) =
              (f32x4){acc[rt][dm][4 * c], acc[rt][dm][4 * c + 1], acc[rt][dm][4 * c + 2],
                      acc[rt][dm][4 * c + 3]};
        }
      for (int k = lane; k < 32 * CR; k += 64) {
        const int row = k / CR, ch = k % CR, r = w0 + 32 * rt + row;
        if (r >= R || r / a.group >= t) continue;
        const size_t at = ((size_t)e * a.splits + sp) * R + r;
        *reinterpret_cast<f32x4*>(a.opart + at * D + 4 * ch) =
            *reinterpret_cast<const f32x4*>(out + (row * CR + (ch ^ (row & 15))) * 16);
      }
      const int r = w0 + 32 * rt + l32;
      if (h == 0 && r < R && r / a.group < t)
        a.mpart[((size_t)e * a.splits + sp) * R + r] = make_float4(-nref[rt], rsum[rt], sum[rt], 0.f);
    }
  } else {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float inv = rsum[rt] == 0.f ? 0.f : 1.f / rsum[rt];
#pragma unroll
      for (int dm = 0; dm < DM; ++dm)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int ch = 4 * dm + c;   // 8 columns; this lane's half of it
          uint2 w;
          w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(
              (f32x2){acc[rt][dm][4 * c] * inv, acc[rt][dm][4 * c + 1] * inv}, bf16x2));
          w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(
              (f32x2){acc[rt][dm][4 * c + 2] * inv, acc[rt][dm][4 * c + 3] * inv}, bf16x2));
          *reinterpret_cast<uint2*>(out + ((32 * rt + l32) * CPR + (ch ^ (l32 & (CPR - 1)))) * 16 + 8 * h) = w;
        }
      const int r = w0 + 32 * rt + l32, i = r / a.group;
      if (h == 0 && a.lse && r < R && i < t)
        a.lse[((size_t)e * a.group + (r - i * a.group)) * a.tokens + i] =
            sum[rt] == 0.f ? -__builtin_huge_valf() : (__log2f(sum[rt]) - nref[rt]) * kLn2;
    }
    for (int k = lane; k < WR * CPR; k += 64) {
      const int row = k / CPR, ch = k % CPR, r = w0 + row;
      const int i = r / a.group, g = r - i * a.group;
      if (r >= R || i >= t) continue;
      *reinterpret_cast<uint4*>((u16*)a.o + (((size_t)e * a.group + g) * a.tokens + i) * D + 8 * ch) =
          *reinterpret_cast<const uint4*>(out + (row * CPR + (ch ^ (row & (CPR - 1)))) * 16);
    }
  }
}

template <int D>
hipError_t launch_wide_d(const AttendK& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks), th(kWTh);
  if (a.lens) {
    if (a.rows == 128) hipLaunchKernelGGL((wide_kernel<D, 1, true>), grid, th, 0, s, a);
    else hipLaunchKernelGGL((wide_kernel<D, 2, true>), grid, th, 0, s, a);
  } else {
    if (a.rows == 128) hipLaunchKernelGGL((wide_kernel<D, 1, false>), grid, th, 0, s, a);
    else hipLaunchKernelGGL((wide_kernel<D, 2, false>), grid, th, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_wide(const AttendK& a, int d, hipStream_t s) {
  return d == 64 ? launch_wide_d<64>(a, s) : launch_wide_d<128>(a, s);
}

}  // namespace grkv
