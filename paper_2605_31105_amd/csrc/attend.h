// What the attention kernels share: which slots a block's rows see, how blocks
// map to work, and the outputs.
#pragma once

#include "grkv_device.h"
#include "grkv_internal.h"

namespace grkv {

constexpr float kUnset = 3e38f;      // minus the reference of a row without one
// The reference of a row, by kernel.  Few rows (attend.hip): it is set this much (log2) above
// the largest logit so far and moves when a logit passes it, so that no weight is above 1 and
// sums hold whatever those against the largest logit would, values near a float's largest
// included.
constexpr float kRefAbove = 8.f;
// Many rows (attend_wide.hip): it is the largest logit and moves where a step's weights of a
// lane sum to more than this.  Values past 2^128 / 2^16 / keys may then overflow: where a sum
// is not finite and no value is the cause, rows are summed again (rows_by_key).  (A reference
// set above the logits there takes two registers more, 170 of head_dim 64, where 168 leave
// room for a third wave: a 16k prompt with a 4k window 577 -> 630 us.)
constexpr float kMoveLog = 16.f, kMoveSum = 0x1p16f;   // log2 of it, and it
constexpr uint32_t kOnes = 0x3f803f80u;   // two bf16 ones
constexpr float kLn2 = 0.6931471805599453f;

// The slots a block's rows may see, in tiles of TK: tiles 0 .. at - 1 (sinks)
// and bt .. (the window), `nt` in all; `full` slots before `lim` and from `lo` on
// (or among the sinks) are seen by every row.
struct Span {
  int at, bt, nt;
  int kend;        // slots that any row may see end here
  int lim, lo;
  int chunk, ns;   // tiles per split, splits in use
};

__device__ __forceinline__ Span make_span(const AttendK& a, int len, int base, int t, int i0, int i1,
                                          int tk) {
  Span s;
  if (a.lens) {   // drafted tokens i0 .. i1 lie at positions base .. base + t - 1
    s.kend = t > 0 ? len : 0;
    s.lim = base;
    s.lo = base + t - a.window;
  } else {        // query i is position base + i
    s.kend = base + i1 + 1;
    s.lim = base + i0 + 1;
    s.lo = base + i1 + 1 - a.window;
  }
  s.at = s.bt = 0;
  if (a.window > 0) {
    const int first = (a.lens ? base : base + i0) + 1 - a.window;
    s.at = (min(a.n_sink, s.kend) + tk - 1) / tk;
    s.bt = max(first > 0 ? first / tk : 0, s.at);
  } else {
    s.lo = 0;
  }
  const int end = (s.kend + tk - 1) / tk;
  s.nt = s.at + max(0, end - s.bt);
  // (a sink tile past the end: a.n_sink was cut to kend)
  s.chunk = max(a.min_tiles, (s.nt + a.splits - 1) >> a.split_shift);
  s.ns = (s.nt + s.chunk - 1) / s.chunk;
  return s;
}

// r / group for r < 2^31, by the multiplication with a rounded-up reciprocal of
// 32 + gshift bits (its top bit is the addition).
__device__ __forceinline__ int group_of(const AttendK& a, int r) {
  return (int)((__umulhi((uint32_t)r, a.gmul) + (uint32_t)r) >> a.gshift);
}

// Block b's entry, row group and split.  Blocks go round the 8 XCDs in turn: with
// `grouped` the row groups of one split follow one another on one XCD, whose L2
// then reads the keys once (entries x splits rounded up to 8); fewer splits than
// that are dealt out row group by row group, so that no XCD is left idle.
__device__ __forceinline__ bool block_work(const AttendK& a, int* e, int* rg, int* sp) {
  const uint32_t b = blockIdx.x;
  uint32_t w;
  if (a.row_groups == 1) {
    w = b;
    *rg = 0;
  } else if (a.grouped) {
    const uint32_t c = b >> 3;
    w = (c / a.row_groups) * 8 + (b & 7);
    *rg = (int)(c % a.row_groups);
  } else {
    const uint32_t all = (uint32_t)a.entries * a.splits;
    w = b % all;
    *rg = (int)(b / all);
  }
  *sp = (int)(w & (a.splits - 1));   // (a power of two)
  const uint32_t ee = w >> a.split_shift;
  *e = (int)ee;
  return ee < (uint32_t)a.entries;
}

// The length, drafted tokens and table row of entry e.
__device__ __forceinline__ void entry_shape(const AttendK& a, int e, int* len, int* t,
                                            const int32_t** row) {
  if (a.lens) {
    const int u = a.units ? a.units[e] : e;
    const bool ok = (unsigned)u < (unsigned)a.pool_units;
    *len = ok ? min(max(a.lens[u], 0), a.max_pages << a.shift) : 0;
    *row = a.table + (size_t)(ok ? u : 0) * a.max_pages;
    *t = a.counts ? min(max(a.counts[e], 0), a.tokens) : a.tokens;
  } else {
    *len = a.n;
    *t = a.tokens;
    *row = nullptr;
  }
}

// Four values of output row `at`: x / l; lse from the reference m and the sum
// lx of the weights before their rounding.
template <typename E, int D>
__device__ __forceinline__ void write_out(const AttendK& a, size_t at, int ch, f32x4 x, float m,
                                          float l, float lx) {
  x *= l == 0.f ? 0.f : 1.f / l;
  if constexpr (sizeof(E) == 2) {
    uint2 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[0], x[1]}, bf16x2));
    w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2], x[3]}, bf16x2));
    *reinterpret_cast<uint2*>((E*)a.o + at * D + 4 * ch) = w;
  } else {
    *reinterpret_cast<f32x4*>((E*)a.o + at * D + 4 * ch) = x;
  }
  if (ch == 0 && a.lse) a.lse[at] = lx == 0.f ? -__builtin_huge_valf() : (m + __log2f(lx)) * kLn2;
}

// Sums of one split.
struct Split {
  float m, l, lx;   // reference; weights after and before their rounding
  f32x4 x;          // four columns
};

// Parts of splits that the blocks join themselves pass between XCDs inside one
// launch, whose L2 caches are not coherent for plain accesses.  They are written
// and read by atomic accesses of agent scope, which go through to where all XCDs
// meet; a wave's own wait for its stores then orders them.  (Fences of that scope
// write back and invalidate a whole L2: 512 units of 4250 keys, two splits, 457 us
// against 227 with a second launch.)
__device__ __forceinline__ void put64(void* p, uint64_t v) {
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get64(const void* p) {
  return __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void wait_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ void put4(float* p, f32x4 v, bool shared) {
  if (shared) {
    const ulonglong2 w = __builtin_bit_cast(ulonglong2, v);
    put64(p, w.x);
    put64(p + 2, w.y);
  } else {
    *reinterpret_cast<f32x4*>(p) = v;
  }
}
template <bool SHARED>
__device__ __forceinline__ f32x4 get4(const float* p) {
  if constexpr (SHARED) {
    const ulonglong2 w = make_ulonglong2(get64(p), get64(p + 2));
    return __builtin_bit_cast(f32x4, w);
  } else {
    return *reinterpret_cast<const f32x4*>(p);
  }
}

// Adds split `y` to `o`, both against the larger of their references.
__device__ __forceinline__ void add_split(Split& o, const Split& y) {
  const float m = fmaxf(o.m, y.m), f = __builtin_amdgcn_exp2f(o.m - m), fy = __builtin_amdgcn_exp2f(y.m - m);
  o.m = m;
  o.l = o.l * f + y.l * fy;
  o.lx = o.lx * f + y.lx * fy;
  o.x = o.x * f + y.x * fy;
}

// Columns 4 ch .. of a row from splits s0, s0 + step, .. below ns, in that order.  The
// reads of eight splits go out together.  The row is at0 + first in split 0 and at0 + s *
// stride in split s > 0.
template <int D, bool SHARED>
__device__ __forceinline__ Split add_splits(const AttendK& a, size_t at0, int first, int stride, int ns,
                                            int s0, int step, int ch) {
  constexpr int B = 8;
  Split o = {-kUnset, 0.f, 0.f, zero4()};
  for (; s0 < ns; s0 += B * step) {
    f32x4 ml[B], x[B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const int s = s0 + k * step;
      ml[k] = (f32x4){-kUnset, 0.f, 0.f, 0.f};
      x[k] = zero4();
      if (s < ns) {
        const size_t at = at0 + (s == 0 ? (size_t)first : (size_t)s * stride);
        ml[k] = get4<SHARED>((const float*)(a.mpart + at));
        x[k] = get4<SHARED>(a.opart + at * D + 4 * ch);
      }
    }
    float m = o.m;
#pragma unroll
    for (int k = 0; k < B; ++k) m = fmaxf(m, ml[k][0]);
    const float f0 = __builtin_amdgcn_exp2f(o.m - m);
    o = {m, o.l * f0, o.lx * f0, o.x * f0};
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const float f = __builtin_amdgcn_exp2f(ml[k][0] - m);
      o.l += ml[k][1] * f;
      o.lx += ml[k][2] * f;
      o.x += x[k] * f;
    }
  }
  return o;
}

// Whether this block is one that finds all `ns` splits of its row group written:
// the last to finish, or another that finishes with it (they write the same
// rows).  Every block marks its split with the call's nonce once its parts are
// out, and reads all marks once its own is: of two blocks one sees the other's.  A
// block that sees them all puts them back to zero, so that a captured call finds
// no marks of its last replay; what else the workspace held does not equal a nonce
// of 64 bits.
__device__ __forceinline__ bool splits_done(const AttendK& a, size_t group, int sp, int ns) {
  __shared__ int done_s;
  wait_stores();   // every wave's part is out
  __syncthreads();
  uint64_t* f = a.flags + group * a.splits;
  if (threadIdx.x < 64) {
    if (threadIdx.x == 0) put64(f + sp, a.nonce);
    wait_stores();
    const bool all = __all((int)threadIdx.x >= ns || get64(f + threadIdx.x) == a.nonce);
    if (all && (int)threadIdx.x < ns) put64(f + threadIdx.x, 0);
    if (threadIdx.x == 0) done_s = all;
  }
  __syncthreads();
  return done_s != 0;
}

// What this lane's row sees: slots before lim from lo on or below n_sink, and
// with pages the drafted tokens of `bits` (slot base + n is bit n).
struct RowSight {
  int lim, lo;
  uint64_t bits;
};

template <bool PAGED>
__device__ __forceinline__ bool sees(const RowSight& s, int j, int n_sink, int base, int len) {
  bool on = j < s.lim && (j >= s.lo || j < n_sink);
  if (PAGED) {
    const int n = j - base;
    on |= n >= 0 && n < 64 && j < len && (s.bits >> (n & 63) & 1) != 0;
  }
  return on;
}

// The same of slots slot0 .. slot0 + 31, a bit each.
template <bool PAGED>
__device__ __forceinline__ uint32_t sees32(const RowSight& s, int slot0, int n_sink, int base, int len) {
  auto below = [&](int end) {   // the slots before `end`
    const int n = end - slot0;
    return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u;
  };
  uint32_t on = below(s.lim) & (~below(s.lo) | below(n_sink));
  if (PAGED) {
    const int n = slot0 - base;   // drafted token of the first of them
    const uint32_t d = n >= 64 || n <= -32 ? 0u
                       : n >= 0 ? (uint32_t)(s.bits >> n) : (uint32_t)(s.bits << -n);
    on |= d & below(len) & ~below(0);
  }
  return on;
}

// Drafted token `lane` of entry e: its ancestors and itself (a bit per token) as
// far as it sees them, and its depth, by doubling the step from a token to its
// parent.  Every lane of the wave takes part.
__device__ __forceinline__ void draft_family(const AttendK& a, int e, int t, int base, int lane,
                                             uint64_t* bits, int* depth) {
  uint64_t family = 1ull << lane;
  *depth = 0;
  if (a.tokens > 1) {
    const int up = lane >= t ? -1
                   : a.parents ? a.parents[(size_t)(e / a.per_tree) * a.tokens + lane] : lane - 1;
    int at = up >= 0 && up < lane ? up : -1;   // (any other parent counts as none)
#pragma unroll
    for (int k = 0; k < 6; ++k) {
      const uint64_t f = __shfl((unsigned long long)family, at & 63);
      const int next = __shfl(at, at & 63);
      if (at >= 0) {
        family |= f;
        at = next;
      }
    }
    *depth = __popcll(family) - 1;
    if (a.window > 0 && a.window < t) {
      // ancestors that have left the window (and are not sinks)
      uint64_t in = 0;
      for (int j = 0; j < t; ++j) {
        const int dj = __builtin_amdgcn_readlane(*depth, j);
        if (*depth - dj < a.window || base + dj < a.n_sink) in |= 1ull << j;
      }
      family &= in;
    }
  }
  *bits = family;
}

// The row of (query i, head) with drafted token i's family and depth held by
// lane i.
template <bool PAGED>
__device__ __forceinline__ RowSight row_sight(const AttendK& a, int base, int i, bool on,
                                              uint64_t family, int depth) {
  RowSight s;
  int pos = base + i;
  s.bits = 0;
  if (PAGED) {
    const uint64_t f = __shfl((unsigned long long)family, i & 63);
    pos = base + __shfl(depth, i & 63);
    if (on) s.bits = f;
  }
  s.lim = on ? (PAGED ? base : pos + 1) : 0;
  s.lo = a.window > 0 ? pos + 1 - a.window : 0;
  return s;
}

// Whether a tile of vt0 .. vt1 - 1 that is not seen whole (by every row before lim and
// from lo on; lim 0: any tile) holds an infinity or NaN among its values.  One wave; asked
// only where a sum of values is not finite.
template <typename E, int D, bool PAGED>
__device__ __forceinline__ bool odd_values(const AttendK& a, const Span& sn, int e, int vt0, int vt1,
                                           int tk, int lim, int lo, const int32_t* trow) {
  constexpr int CPR = D * (int)sizeof(E) / 16;   // 16-byte chunks of a row
  const int lane = threadIdx.x & 63;
  for (int vt = vt0; vt < vt1; ++vt) {
    const int slot0 = (vt < sn.at ? vt : vt - sn.at + sn.bt) * tk;
    if (slot0 + tk <= lim && (slot0 >= lo || slot0 + tk <= a.n_sink)) continue;
    bool odd = false;
#pragma unroll 4
    for (int k = lane; k < tk * CPR; k += 64) {
      const int j = slot0 + k / CPR;
      if (j >= sn.kend) continue;
      size_t row = (size_t)e * a.n + j;
      if (PAGED) {
        const int p = trow[j >> a.shift];
        row = ((size_t)((unsigned)p < (unsigned)a.pages ? p : 0) << a.shift) + (j & ((1 << a.shift) - 1));
      }
      const uint4 x = *reinterpret_cast<const uint4*>((const E*)a.v + row * D + k % CPR * (16 / sizeof(E)));
      for (const uint32_t w : {x.x, x.y, x.z, x.w}) {
        odd |= (w & 0x7f800000u) == 0x7f800000u;
        if constexpr (sizeof(E) == 2) odd |= (w & 0x7f80u) == 0x7f80u;
      }
    }
    if (__any(odd)) return true;
  }
  return false;
}

// Whether a row's weights left float32's reach: of logits past 2^30, whose step is many powers
// of two, the largest may lie far from its own reference, on either side.
__device__ __forceinline__ bool far_off(float sum, float nref) {
  return sum > 0x1p40f || (sum < 0x1p-60f && nref != kUnset);
}

// Rows of a split once more, key by key, with float32 weights against the largest logit:
// taken where an infinity or NaN among the values of a tile that is not seen whole may have
// reached rows that do not see it (0 x inf in a product is NaN), where large values overflowed
// under a reference that was too low, and where weights are far off.  One wave; rows first ..
// first + count - 1 of entry e over tiles vt0 .. vt1 - 1 of sn, left as partial rows
// from `part` on or (part < 0) as outputs.  A lane forms the weight of one key of 64, then
// sums D / 64 columns.
template <typename E, int D, bool PAGED>
__device__ __forceinline__ void rows_by_key(const AttendK& a, const Span& sn, int e, int64_t part, int first,
                                            int count, int vt0, int vt1, int tk, int len, int t,
                                            const int32_t* trow, uint64_t family, int depth) {
  constexpr bool BF = sizeof(E) == 2;
  constexpr int C = D / 64;
  const int lane = threadIdx.x & 63, R = a.group * a.tokens, base = len - t;
  auto value = [](E x) -> float {
    if constexpr (sizeof(E) == 2) return bf16_to_f32(x);
    else return x;
  };
  auto slot_row = [&](int slot) -> size_t {
    if (!PAGED) return (size_t)e * a.n + slot;
    const int p = trow[slot >> a.shift];
    return ((size_t)((unsigned)p < (unsigned)a.pages ? p : 0) << a.shift) + (slot & ((1 << a.shift) - 1));
  };
  for (int n = 0; n < count; ++n) {
    const int r = first + n, i = group_of(a, r), g = r - i * a.group;
    if (r >= R) return;
    const RowSight sight = row_sight<PAGED>(a, base, i, i < t, family, depth);
    const size_t at = ((size_t)e * a.group + g) * a.tokens + i;
    if (i >= t) continue;
    const E* q = (const E*)a.q + at * D;
    float m = -kUnset, l = 0.f, o[C] = {};
    for (int vt = vt0; vt < vt1; ++vt) {
      const int slot0 = (vt < sn.at ? vt : vt - sn.at + sn.bt) * tk;
      for (int j0 = slot0; j0 < slot0 + tk; j0 += 64) {
        const int j = j0 + lane;
        const bool on = j < slot0 + tk && j < sn.kend && sees<PAGED>(sight, j, a.n_sink, base, len);
        float x = -__builtin_huge_valf();
        if (on) {
          const E* k = (const E*)a.k + slot_row(j) * D;
          x = 0.f;
          for (int c = 0; c < D; ++c) x = fmaf(value(q[c]), value(k[c]), x);
          x *= a.scale_log2;
        }
        float mx = x;
        for (int k = 1; k < 64; k <<= 1) mx = fmaxf(mx, __shfl_xor(mx, k));
        if (mx > m) {
          const float f = __builtin_amdgcn_exp2f(m - mx);
          m = mx;
          l *= f;
          for (int c = 0; c < C; ++c) o[c] *= f;
        }
        const float w = on ? __builtin_amdgcn_exp2f(x - m) : 0.f;
        float s = w;
        for (int k = 1; k < 64; k <<= 1) s += __shfl_xor(s, k);
        l += s;
        for (int k = 0; k < 64; ++k) {
          const float wk = __shfl(w, k);
          if (!__shfl((int)on, k)) continue;
          const E* v = (const E*)a.v + slot_row(j0 + k) * D;
          for (int c = 0; c < C; ++c) o[c] = fmaf(wk, value(v[64 * c + lane]), o[c]);
        }
      }
    }
    if (part >= 0) {
      const size_t to = part + r;
      for (int c = 0; c < C; ++c)
        __hip_atomic_store(a.opart + to * D + 64 * c + lane, o[c], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (lane == 0) put4((float*)(a.mpart + to), (f32x4){m, l, l, 0.f}, true);
    } else {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      for (int c = 0; c < C; ++c) {
        E* to = (E*)a.o + at * D + 64 * c + lane;
        if constexpr (BF) *reinterpret_cast<__bf16*>(to) = (__bf16)(o[c] * inv);
        else *to = o[c] * inv;
      }
      if (lane == 0 && a.lse) a.lse[at] = l == 0.f ? -__builtin_huge_valf() : (m + __log2f(l)) * kLn2;
    }
  }
}

}  // namespace grkv
