// Attention of many query rows over the keys of a unit (bf16): prompts and chunks
// of them with a window and sinks, trees of drafted tokens with more than 64 rows
// (attend_plan in attend.hip says from where on).
//
// The sums are those of attend.hip; here the products and the exponentials bound
// them, so the four waves of a block share tiles of 64 keys in LDS:
//  * A wave holds 32 rows and forms, in one step, the weights of 64 keys beside the
//    logits of the next 64, then P.V.  Two blocks share a compute unit, and the wave of
//    the other one on its SIMD fills the gaps.  (8 units of 4 heads, a 16k prompt with a
//    4k window: 955 to 1015 us beside 1374 of one wave of 64 rows per SIMD, which
//    reads half as much LDS but waits for its own chain of logit, exponential and
//    product.  One block of eight waves and 256 rows: 969, and with head_dim 64 476
//    beside 402, since its waves meet at one barrier.)
//  * K and V go from memory to LDS (global_load_lds): two K tiles and two V tiles, K one
//    step ahead of V, one barrier per tile.  16-byte chunks are permuted by row so that
//    neither the K operand reads nor the V transpose reads conflict.
//  * 32x32x16 MFMAs: S^T = K Q^T leaves a query row in each lane column, where
//    P^T already is the B operand of O^T = V^T P^T.
//  * References, rounding and values that are not finite: as in attend.hip, but that
//    a step looks for a row's largest logit only where its sum of weights passes 2^16.
//  * P is rounded to bf16 (2^-8 of a weight), and o divided by the sum of the rounded weights
//    (dot products with ones), so that the weights of a row add up to one; lse comes from
//    the sum before the rounding.  A second product with what the rounding leaves, as in
//    attend.hip, would cost what bounds these calls: a 16k prompt with a 4k window 995 -> 1300
//    us (head_dim 64 595 -> 790), trees of 32 over 32k keys 109 -> 123, 8 prompts of 1000 25.3
//    -> 29.6.  (The error of o against 64 bits, rounded to bf16 as it is, falls from 0.0022
//    to 0.0017 of its norm.)
#include "attend.h"

namespace grkv {
namespace {

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

template <int D, bool PAGED>
__global__ __launch_bounds__(kWTh, 2) void wide_kernel(AttendK a) {
  constexpr int TK = kWideKeys;
  constexpr int NK = TK / 32;          // 32-key parts of a step
  constexpr int RB = 2 * D;            // bytes of a row
  constexpr int CPR = RB / 16;         // chunks of a row
  constexpr int KB = TK * RB;          // bytes of a K (or V) tile
  constexpr int NI = 16 * RB / 1024;   // load instructions per wave and tensor: 16 rows
  constexpr int RPI = 64 / CPR;        // rows of one
  constexpr int KS = D / 16, DM = D / 32;
  static_assert(TK == 16 * kWWaves, "a wave brings 16 rows of a tile");
  static_assert(kWWaves * 32 * D * 4 == 4 * KB, "the waves' outputs fit the ring");
  __shared__ __attribute__((aligned(1024))) char ring[4 * KB];   // two K tiles, two V tiles

  int e, rg, sp;
  if (!block_work(a, &e, &rg, &sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int R = a.group * a.tokens, r0 = rg * a.rows;
  int len, t;
  const int32_t* trow;
  entry_shape(a, e, &len, &t, &trow);
  const int base = len - t;
  const Span sn = make_span(a, len, base, t, group_of(a, r0), group_of(a, min(r0 + a.rows - 1, R - 1)), TK);
  const int vt0 = sp * sn.chunk, vt1 = min(sn.nt, vt0 + sn.chunk);
  if (sp > 0 && vt0 >= sn.nt) return;

  uint64_t family = 0;
  int depth = 0;
  if (PAGED) draft_family(a, e, t, base, lane, &family, &depth);
  const int w0 = r0 + 32 * wave;   // this wave's first row
  bf16x8 qf[KS];
  RowSight sight;
  {
    const int r = w0 + l32;
    const int i = group_of(a, r), g = r - i * a.group;
    const bool on = r < R && i < t;
    sight = row_sight<PAGED>(a, base, i, on, family, depth);
    const u16* q = (const u16*)a.q + (((size_t)e * a.group + g) * a.tokens + i) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (on) qf[ks] = *reinterpret_cast<const bf16x8*>(q + 16 * ks + 8 * h);
      else qf[ks] = bf16x8{};
    }
  }
  // slots that every row of the wave sees: before lim and from lo on, or sinks
  int lim = sn.lim, lo = sn.lo;
  if (!PAGED) {
    lim = base + group_of(a, min(w0, R - 1)) + 1;
    lo = a.window > 0 ? base + group_of(a, min(w0 + 31, R - 1)) + 1 - a.window : 0;
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
  // this wave's rows of tile vt, of K or V (the chunk offsets o, permuted by swz)
  auto load = [&](const void* from, int vt, int to, const uint32_t (&o)[NI], auto swz, bool once)
                  __attribute__((always_inline)) {
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
    const char* src = (const char*)from + row * RB;
    const uint32_t dst = __builtin_amdgcn_readfirstlane(ring0 + to + wave * 16 * RB);
    const bool whole = s16 + 15 <= last;
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      uint32_t f = o[it];
      if (!whole) {   // rows past the last slot: the last one again
        const int row_in = it * RPI + lane / CPR, ch = lane % CPR;
        f = ((min(s16 + row_in, last) & 15) * CPR + (ch ^ swz(row_in))) * 16;
      }
      if (once) ring_load<true>(src, f, dst + it * 1024);
      else ring_load(src, f, dst + it * 1024);
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

  f32x16 acc[DM], st[NK];
  float nref = kUnset;          // minus the reference
  float sum = 0.f, rsum = 0.f;  // weights' sums before and after their rounding (this lane's keys)
#pragma unroll
  for (int dm = 0; dm < DM; ++dm) acc[dm] = f32x16{};

  auto logits = [&](const char* kt, f32x16 (&x)[NK]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      bf16x8 kf[KS];
      read_k(kt + n * 32 * RB, kf);
      x[n] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x[n] = mfma32(kf[ks], qf[ks], x[n]);
    }
  };
  // One step: the 32 NK keys at slot0, whose logits are in st and whose V rows are at vt;
  // kt: K rows of the next step.
  auto step = [&](int slot0, const char* kt, const char* vt) __attribute__((always_inline)) {
    const bool full = slot0 + 32 * NK <= lim && (slot0 >= lo || slot0 + 32 * NK <= a.n_sink);
    if (!full) {
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        const uint32_t on = sees32<PAGED>(sight, slot0 + 32 * n, a.n_sink, base, len) >> (4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((on >> (8 * (r / 4) + r % 4) & 1) == 0) st[n][r] = -__builtin_huge_valf();
      }
    }
    f32x16 nx[NK];
    logits(kt, nx);
    bf16x8 p[NK][2];
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
            const bf16x2 w = __builtin_convertvector((f32x2){x0, x1}, bf16x2);
            p[n][s][c] = w[0];
            p[n][s][c + 1] = w[1];
            s2 = __builtin_amdgcn_fdot2_f32_bf16(w, __builtin_bit_cast(bf16x2, kOnes), s2, false);
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
      read_v(vt + n * 32 * RB, vf);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int dm = 0; dm < DM; ++dm) acc[dm] = mfma32(vf[s][dm], p[n][s], acc[dm]);
    }
#pragma unroll
    for (int n = 0; n < NK; ++n) st[n] = nx[n];
  };

  if (vt0 < vt1) {
    // values that no other row group reads are read once (32 units of 20k to 32k keys,
    // over caches used in turn, 116 -> 114 us; keys too, 114)
    const bool once = PAGED && a.row_groups == 1;
    // K of tile i is in half i & 1 of the first half of the ring, V in the second
    auto load_k = [&](int i) { load(a.k, min(vt0 + i, vt1 - 1), (i & 1) * KB, ko, swz_k, false); };
    auto load_v = [&](int i) { load(a.v, min(vt0 + i, vt1 - 1), (2 + (i & 1)) * KB, vo, swz_v, once); };
    load_k(0);
    load_k(1);
    load_v(0);
    ring_barrier<2 * NI>();
    logits(ring, st);
    for (int i = 0; i < vt1 - vt0; ++i) {
      // K of tile i + 1 and V of tile i are here, and every wave is done with K of
      // tile i and V of tile i - 1
      ring_barrier<0>();
      load_k(i + 2);
      load_v(i + 1);
      step(slot_of(vt0 + i), ring + ((i + 1) & 1) * KB, ring + (2 + (i & 1)) * KB);
    }
  }
  ring_barrier<0>();   // (the ring is the output's buffer now)
  sum += __shfl_xor(sum, 32);
  rsum += __shfl_xor(rsum, 32);
  float odd = 0.f;   // NaN if a sum of values is not finite
#pragma unroll
  for (int dm = 0; dm < DM; ++dm)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(acc[dm][r], 0.f, odd);
  const int64_t part = ((int64_t)e * a.splits + sp) * R;
  const bool far = far_off(sum, nref);
  if (__any(far || (odd != odd && sum == sum)) &&
      (__any(far) || odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, lim, lo, trow) ||
       !odd_values<u16, D, PAGED>(a, sn, e, vt0, vt1, TK, 0, lo, trow))) {
    if (PAGED) draft_family(a, e, t, base, lane, &family, &depth);   // (not held until here)
    rows_by_key<u16, D, PAGED>(a, sn, e, sn.ns > 1 ? part : -1, w0, 32, vt0, vt1, TK, len, t, trow, family, depth);
    return;
  }
  // a wave's rows through its part of the ring (lane's four columns 32 dm + 8 c + 4 h of
  // row l32, chunks permuted by row), so that they leave whole
  const int my = w0 + l32, mi = group_of(a, my);
  char* out = ring + wave * KB;
  if (sn.ns > 1) {
    constexpr int CR = D / 4;
    const float fit = 1.f / kMoveSum;   // (weights of 1 at most, so that parts may be added)
#pragma unroll
    for (int dm = 0; dm < DM; ++dm)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<f32x4*>(out + (l32 * CR + ((8 * dm + 2 * c + h) ^ (l32 & 15))) * 16) =
            (f32x4){acc[dm][4 * c], acc[dm][4 * c + 1], acc[dm][4 * c + 2], acc[dm][4 * c + 3]} * fit;
    if (h == 0 && my < R && mi < t)
      a.mpart[part + my] = make_float4(kMoveLog - nref, rsum * fit, sum * fit, 0.f);
#pragma unroll 4
    for (int k = lane; k < 32 * CR; k += 64) {
      const int row = k / CR, ch = k % CR, r = w0 + row;
      if (r < R && group_of(a, r) < t)
        *reinterpret_cast<f32x4*>(a.opart + (part + r) * D + 4 * ch) =
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
  auto place = [&](int r, int i) { return ((size_t)e * a.group + (r - i * a.group)) * a.tokens + i; };
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

template <int D>
hipError_t launch_wide_d(const AttendK& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks), th(kWTh);
  if (a.lens) hipLaunchKernelGGL((wide_kernel<D, true>), grid, th, 0, s, a);
  else hipLaunchKernelGGL((wide_kernel<D, false>), grid, th, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_wide(const AttendK& a, int d, hipStream_t s) {
  return d == 64 ? launch_wide_d<64>(a, s) : launch_wide_d<128>(a, s);
}

}  // namespace grkv
