// What the plans of calls on pages share (one block each): scans and the handing out
// of free pages.
#pragma once

#include "grkv_device.h"
#include "grkv_internal.h"

namespace grkv {

constexpr int kPlanTh = 1024;
constexpr int kNoOwner = 0x7fffffff;
constexpr int kOwnerUnits = 8192;   // units of a pool whose owners fit the plan's LDS

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

// The lowest free pages of the pool, `want` of them or as many as there are, into ids in
// order; their bits are cleared.  bits0: this thread's word of the bitmap, read before.
// A thread takes a word of 32 pages; the numbers are written two words at a time by a wave,
// neighbouring lanes neighbouring numbers, the waves in turn (plans of 2048 and 34k pages
// 6.3 and 12.4 us; each wave the words that its lanes hold, 10.1 and 19.2)
__device__ __forceinline__ uint32_t take_pages(const grkv_pages& pg, uint32_t want, uint32_t bits0,
                                               int32_t* ids, int* turn) {
  __shared__ uint32_t scratch32[2][kPlanTh / 64];
  __shared__ uint32_t taken_s[kPlanTh], rank_s[kPlanTh];   // pages taken of a word, the first one's rank
  const int tid = threadIdx.x, lane = tid & 63, words = (pg.pages + 31) / 32;
  uint32_t found = 0;
  for (int w0 = 0; w0 < words && found < want; w0 += kPlanTh) {
    const int w = w0 + tid;
    const uint32_t bits = w0 == 0 ? bits0 : w < words ? pg.free_bits[w] : 0u;
    uint32_t total;
    const uint32_t r0 = found + plan_scan((uint32_t)__popc(bits), scratch32, (*turn)++, &total);
    uint32_t left = 0;
    if (r0 + __popc(bits) > want) {   // the last word taken from, and those behind it
      left = bits;
      for (uint32_t r = r0; r < want; ++r) left &= left - 1;
    }
    if (left != bits) pg.free_bits[w] = left;
    taken_s[tid] = bits ^ left;
    rank_s[tid] = r0;
    __syncthreads();   // (read before the next scan's barrier)
    const int here = min(words - w0, kPlanTh), bit = lane & 31;
    for (int k = (tid >> 6) * 2 + (lane >> 5); k < here; k += kPlanTh / 32) {
      const uint32_t t = taken_s[k];
      if (t >> bit & 1) ids[rank_s[k] + __popc(t & ((1u << bit) - 1))] = 32 * (w0 + k) + bit;
    }
    found += total;
  }
  return found < want ? found : want;
}

}  // namespace grkv
