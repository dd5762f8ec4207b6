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
#include "wide_rows.h"

namespace grkv {
namespace {

// (head_dim 64 over contiguous keys: 168 registers, three waves per SIMD)
template <int D, Rows KIND>
__global__ __launch_bounds__(kWTh, D == 64 && KIND == kContiguous ? 3 : 2) void wide_kernel(AttendK a) {
  __shared__ __attribute__((aligned(1024))) char ring[2 * kRing<D>];
  int e, rg, sp;
  if (!block_work(a, &e, &rg, &sp)) return;
  const int R = a.group * a.tokens, r0 = rg * a.rows;
  int len, t;
  const int32_t* trow;
  entry_shape(a, e, &len, &t, &trow);
  const Span sn = make_span(a, KIND == kTree, len, len - t, t, group_of(a, r0),
                            group_of(a, min(r0 + a.rows - 1, R - 1)), kWideKeys);
  const int vt0 = sp * sn.chunk, vt1 = min(sn.nt, vt0 + sn.chunk);
  if (sp > 0 && vt0 >= sn.nt) return;
  const auto part = [&] { return Part{sn.ns > 1, ((int64_t)e * a.splits + sp) * R}; };
  wide_rows<D, KIND>(a, sn, e, r0, vt0, vt1, part, len, t, trow, ring, ring + kRing<D>);
}

template <int D>
hipError_t launch_wide_d(const AttendK& a, hipStream_t s) {
  const dim3 grid((unsigned)a.blocks), th(kWTh);
  if (a.lens) hipLaunchKernelGGL((wide_kernel<D, kTree>), grid, th, 0, s, a);
  else hipLaunchKernelGGL((wide_kernel<D, kContiguous>), grid, th, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_wide(const AttendK& a, int d, hipStream_t s) {
  return d == 64 ? launch_wide_d<64>(a, s) : launch_wide_d<128>(a, s);
}

}  // namespace grkv
