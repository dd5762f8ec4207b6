// The units of a step's sequences grown by their new tokens, with every token's position
// and slots (grkv_pages_extend).
//
//   n1 = n0 + c,  pages ceil(n0 / p) .. ceil(n1 / p) - 1 new,  slot of row s = T_u[s / p] p + s % p.
//
// A plan by one block, since which pages a unit gets depends on all units before it, and a
// map by many: a thread per token and head finds its sequence among the starts, writes the
// slot, and where the slot is a page's first, the unit's table and the page's count.  What
// bounds both is the chain of dependent reads and the two launches; the map's 8 bytes per
// token and head are far from HBM's rate.  (A token for 32 sequences of 256 units: plan 19 us, map
// 4; 24 prompts of 8 units that take 18k pages: 12 and 4.)
#include <type_traits>

#include "pages.h"

namespace grkv {
namespace {

constexpr int kMapTh = 256;
constexpr int kAhead = 8;

struct ExtendK {
  grkv_pages pg;
  int shift;                // log2 page_size
  int sequences, heads, entries, tokens;
  const int32_t* units;
  int64_t unit_stride;
  const int32_t* counts;
  const int32_t* seen;
  int32_t* starts;
  int32_t* positions;
  int64_t* slots;
  int32_t* status;
  int32_t* owner;           // [pool units] lowest entry that names the unit
  int32_t* code;            // [sequences] GRKV_PAGES_ of each
  int32_t* first;           // [sequences] position of the first new token
  uint32_t hmul;            // division by heads: see sequence_at
  int hshift;
  int2* jobs;               // [entries] rows before, place of the first new page among ids
  int32_t* ids;             // [pages] pages handed out, in order
};

__device__ __forceinline__ int unit_of(const ExtendK& a, int b, int h) {
  return a.units ? a.units[b * a.unit_stride + h] : b * a.heads + h;
}
// The sequence of entry e (e / heads), by the multiplication with a rounded-up reciprocal of 32 +
// hshift bits (its top bit is the addition).
__device__ __forceinline__ int sequence_at(const ExtendK& a, int e) {
  return (int)((__umulhi((uint32_t)e, a.hmul) + (uint32_t)e) >> a.hshift);
}
// Inclusive sum over the lanes of a wave up to this one, by DPP: within 16 lanes, then the last of
// a row to the next row, and of the first half to the second.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  auto step = [](uint32_t v, auto ctrl, auto rows) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  constexpr std::integral_constant<int, 0xF> all{};
  x = step(x, std::integral_constant<int, 0x111>{}, all);
  x = step(x, std::integral_constant<int, 0x112>{}, all);
  x = step(x, std::integral_constant<int, 0x114>{}, all);
  x = step(x, std::integral_constant<int, 0x118>{}, all);
  x = step(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});
  return step(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
}
__device__ __forceinline__ int count_of(const ExtendK& a, int b) { return max(a.counts[b], 0); }
__device__ __forceinline__ int pages_of(const ExtendK& a, int64_t rows) {
  return (int)((rows + (1 << a.shift) - 1) >> a.shift);
}

__global__ __launch_bounds__(kPlanTh) void extend_plan_kernel(ExtendK a) {
  __shared__ int owner_s[kOwnerUnits];
  __shared__ unsigned long long scratch[2][kPlanTh / 64];
  constexpr int WAVES = kPlanTh / 64;
  static_assert(kAhead * WAVES == 128, "two sums to a lane");
  __shared__ unsigned long long sums_s[kAhead * WAVES + 1];
  __shared__ int used_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t cap = (int64_t)a.pg.max_pages << a.shift;
  auto in_pool = [&](int u) { return (unsigned)u < (unsigned)a.pg.units; };
  auto refuse = [&](int b, int code) { atomicMax(a.code + b, code); };
  const uint32_t bits0 = tid < (a.pg.pages + 31) / 32 ? a.pg.free_bits[tid] : 0u;
  int turn = 0;

  // sequences: where their rows start, and their first position
  if (tid == 0) used_s = 0;
  unsigned long long rows = 0;
  bool late = false;   // a sequence of this thread's is refused
  for (int b0 = 0; b0 < a.sequences; b0 += kPlanTh) {
    const int b = b0 + tid;
    const bool on = b < a.sequences;
    const int c = on ? count_of(a, b) : 0;
    unsigned long long total;
    const unsigned long long at = rows + plan_scan((unsigned long long)c, scratch, turn++, &total);
    rows += total;
    if (!on) continue;
    int first = 0;
    if (a.seen) {
      first = a.seen[b];
    } else {
      const int u = unit_of(a, b, 0);
      if (in_pool(u)) first = a.pg.lens[u];   // (a bad length is found below)
    }
    const bool fits = c == 0 || (at + c <= (unsigned long long)a.tokens && first >= 0 && first <= 0x7fffffff - c);
    late |= !fits;
    a.starts[b] = (int)(at < (unsigned)a.tokens ? at : (unsigned)a.tokens);
    a.first[b] = first;
    __hip_atomic_store(a.code + b, fits ? GRKV_PAGES_OK : GRKV_PAGES_RANGE, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  }
  if (tid == 0) a.starts[a.sequences] = (int)(rows < (unsigned)a.tokens ? rows : (unsigned)a.tokens);

  // owner of a unit: the lowest entry that names it
  const bool small = a.pg.units <= kOwnerUnits;
  if (a.units) {
    if (small) {
      for (int u = tid; u < a.pg.units; u += kPlanTh) owner_s[u] = kNoOwner;
    } else {
      for (int e = tid; e < a.entries; e += kPlanTh) {
        const int b = sequence_at(a, e), u = unit_of(a, b, e - b * a.heads);
        if (in_pool(u)) __hip_atomic_store(a.owner + u, kNoOwner, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    __syncthreads();
    for (int e = tid; e < a.entries; e += kPlanTh) {
      const int b = sequence_at(a, e), u = unit_of(a, b, e - b * a.heads);
      if (in_pool(u)) atomicMin(small ? owner_s + u : a.owner + u, e);
    }
  }
  __syncthreads();

  // Entries kAhead to a thread at a time, neighbouring threads' neighbours: their reads go out
  // together, and a barrier serves the scans of all (8192 units 27 -> 19 us).
  constexpr int BATCH = kPlanTh * kAhead;
  auto each = [&](int e0, auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k * kPlanTh + tid;
      if (e0 + k * kPlanTh < a.entries && e < a.entries) f(k, e, sequence_at(a, e));
    }
  };

  // whether each can grow
  bool bad = late;
  for (int e0 = 0; e0 < a.entries; e0 += BATCH) {
    int n[kAhead], c[kAhead], u[kAhead];
    each(e0, [&](int k, int e, int b) { u[k] = unit_of(a, b, e - b * a.heads); });
    each(e0, [&](int k, int, int b) {
      c[k] = count_of(a, b);
      n[k] = in_pool(u[k]) ? a.pg.lens[u[k]] : 0;
    });
    each(e0, [&](int k, int e, int b) {
      int code = GRKV_PAGES_OK;
      if (!in_pool(u[k]) || (a.units && (small ? owner_s[u[k]] : load_agent(a.owner + u[k])) != e) ||
          n[k] < 0 || n[k] > cap)
        code = GRKV_PAGES_UNIT;
      else if ((int64_t)n[k] + c[k] > cap)
        code = GRKV_PAGES_LENGTH;
      if (code != GRKV_PAGES_OK) {
        refuse(b, code);
        bad = true;
      }
      a.jobs[e].x = n[k];
    });
  }
  const bool any = __syncthreads_or(bad);   // a sequence is refused

  // the pages that each needs, and those of the entries before it
  unsigned long long all = 0;
  for (int e0 = 0; e0 < a.entries; e0 += BATCH) {
    // (32 bits hold all needs together: rows that are accepted are tokens * heads < 2^31 in all, in pages
    // of 16 rows or more, and each of the 2^24 entries may begin one page besides)
    uint32_t need[kAhead], before[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) need[k] = 0;
    each(e0, [&](int k, int e, int b) {
      const int n0 = a.jobs[e].x;
      if (!any || load_agent(a.code + b) == GRKV_PAGES_OK)
        need[k] = pages_of(a, (int64_t)n0 + count_of(a, b)) - pages_of(a, n0);
    });
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      before[k] = e0 + k * kPlanTh < a.entries ? wave_scan(need[k]) : 0;
      if (lane == 63) sums_s[k * WAVES + wave] = before[k];
      before[k] -= need[k];
    }
    __syncthreads();
    // (of the batch's waves, in the order of their entries: two to a lane of the first wave)
    if (wave == 0) {
      const unsigned long long x = sums_s[2 * lane], y = sums_s[2 * lane + 1];
      unsigned long long incl = x + y;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned long long t = __shfl_up(incl, d);
        if (lane >= d) incl += t;
      }
      sums_s[2 * lane] = incl - x - y;
      sums_s[2 * lane + 1] = incl - y;
      if (lane == 63) sums_s[kAhead * WAVES] = incl;
    }
    __syncthreads();
    each(e0, [&](int k, int e, int) {
      const unsigned long long off = all + sums_s[k * WAVES + wave] + before[k];
      a.jobs[e].y = (int)(off < (unsigned)a.pg.pages ? off : (unsigned)a.pg.pages);
    });
    all += sums_s[kAhead * WAVES];
    __syncthreads();   // (the next batch writes the sums)
  }
  const uint32_t want = (uint32_t)(all < (unsigned)a.pg.pages ? all : (unsigned)a.pg.pages);
  const uint32_t found = take_pages(a.pg, want, bits0, a.ids, &turn);

  // sequences past the free pages are refused: those behind them that need pages are too,
  // so the pages of the others are the first of ids
  auto needs = [&](int2 j, int c) { return pages_of(a, (int64_t)j.x + c) - pages_of(a, j.x); };
  const bool full = all > found;
  if (full) {
    for (int e = tid; e < a.entries; e += kPlanTh) {
      const int b = sequence_at(a, e);
      if (any && load_agent(a.code + b) != GRKV_PAGES_OK) continue;   // (or refused here, by another of its heads)
      const int2 j = a.jobs[e];
      const int need = needs(j, count_of(a, b));
      if (need > 0 && (uint64_t)j.y + need > found) refuse(b, GRKV_PAGES_FULL);
    }
    __syncthreads();
  }
  int used = 0;
  for (int e0 = 0; e0 < a.entries; e0 += BATCH) {
    int2 j[kAhead];
    int u[kAhead], c[kAhead];
    each(e0, [&](int k, int e, int b) {
      j[k] = a.jobs[e];
      u[k] = unit_of(a, b, e - b * a.heads);
      c[k] = count_of(a, b);
    });
    each(e0, [&](int k, int, int b) {
      if ((any || full) && load_agent(a.code + b) != GRKV_PAGES_OK) return;
      const int need = needs(j[k], c[k]);
      if (need > 0) used = max(used, j[k].y + need);
      a.pg.lens[u[k]] = j[k].x + c[k];
    });
  }
  if (a.status)
    for (int b = tid; b < a.sequences; b += kPlanTh) a.status[b] = load_agent(a.code + b);
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) used = max(used, __shfl_xor(used, k));
  if (lane == 0 && used > 0) atomicMax(&used_s, used);
  __syncthreads();
  // pages taken for refused sequences go back
  for (uint32_t r = used_s + tid; r < found; r += kPlanTh)
    atomicOr(a.pg.free_bits + (a.ids[r] >> 5), 1u << (a.ids[r] & 31));
}

// The sequence of row t: the first whose rows end behind it; `sequences` if there is none.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int sequences, int t) {
  int lo = 0, hi = sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kMapTh) void extend_map_kernel(ExtendK a) {
  const uint32_t g = blockIdx.x * kMapTh + threadIdx.x;
  const int t = (int)(g / (uint32_t)a.heads), h = (int)(g - (uint32_t)t * a.heads);
  if (t >= a.tokens) return;
  const int b = sequence_of(a.starts, a.sequences, t);
  int64_t to = -1;
  int pos = GRKV_NO_POSITION;
  if (b < a.sequences && a.code[b] == GRKV_PAGES_OK) {
    const int2 j = a.jobs[b * a.heads + h];
    const int i = t - a.starts[b], slot = j.x + i, ord = slot >> a.shift, mask = (1 << a.shift) - 1;
    const int fresh = pages_of(a, j.x);
    pos = a.first[b] + i;
    int32_t* entry = a.pg.table + (size_t)unit_of(a, b, h) * a.pg.max_pages + ord;
    int page;
    if (ord < fresh) {
      page = *entry;
    } else {
      page = a.ids[j.y + ord - fresh];
      if ((slot & mask) == 0) {
        *entry = page;
        a.pg.refs[page] = 1;
      }
    }
    if ((unsigned)page < (unsigned)a.pg.pages) to = ((int64_t)page << a.shift) + (slot & mask);
  }
  a.slots[g] = to;
  if (h == 0) a.positions[t] = pos;
}

}  // namespace

ExtendLayout extend_layout(const grkv_pages* pg, int sequences, int heads) {
  ExtendLayout l;
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  l.owner = 0;
  l.code = l.owner + up((size_t)pg->units * sizeof(int32_t));
  l.first = l.code + up((size_t)sequences * sizeof(int32_t));
  l.jobs = l.first + up((size_t)sequences * sizeof(int32_t));
  l.ids = l.jobs + up((size_t)sequences * heads * sizeof(int2));
  l.total = l.ids + up((size_t)pg->pages * sizeof(int32_t));
  return l;
}

hipError_t launch_extend(const grkv_pages* pg, const grkv_step* step, const int32_t* counts,
                         const int32_t* seen, int32_t* starts, int32_t* positions, int64_t* slots,
                         int32_t* status, void* workspace, hipStream_t s) {
  ExtendK a = {};
  a.pg = *pg;
  a.shift = __builtin_ctz((unsigned)pg->page_size);
  a.sequences = step->sequences;
  a.heads = step->heads;
  a.entries = step->sequences * step->heads;
  a.tokens = step->tokens;
  a.units = step->units;
  a.unit_stride = step->unit_stride;
  a.counts = counts;
  a.seen = seen;
  a.starts = starts;
  a.positions = positions;
  a.slots = slots;
  a.status = status;
  while ((1ll << a.hshift) < a.heads) ++a.hshift;
  a.hmul = (uint32_t)((((1ull << a.hshift) - (uint64_t)a.heads) << 32) / (uint64_t)a.heads + 1);
  char* ws = (char*)workspace;
  const ExtendLayout lay = extend_layout(pg, step->sequences, step->heads);
  a.owner = (int32_t*)(ws + lay.owner);
  a.code = (int32_t*)(ws + lay.code);
  a.first = (int32_t*)(ws + lay.first);
  a.jobs = (int2*)(ws + lay.jobs);
  a.ids = (int32_t*)(ws + lay.ids);
  hipLaunchKernelGGL(extend_plan_kernel, dim3(1), dim3(kPlanTh), 0, s, a);
  const int64_t all = (int64_t)a.tokens * a.heads;
  if (all > 0)
    hipLaunchKernelGGL(extend_map_kernel, dim3((unsigned)((all + kMapTh - 1) / kMapTh)), dim3(kMapTh), 0, s, a);
  return hipGetLastError();
}

}  // namespace grkv
