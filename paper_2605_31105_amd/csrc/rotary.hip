// Rotary positions (grkv_rotary), and rows rotated on their way into the pages of a
// cache (grkv_pages_store).
//
// Pair i of a head's first `dims` columns, (a, b), at position p is turned by the angle
// p f_i:  a' = s (a cos - b sin),  b' = s (a sin + b cos);  the other way round for the
// inverse, which is also the gradient (the map is linear, s times a rotation).
//
//  * Angles: p f_i has an absolute error of half a step of its own size in float32, 0.03
//    radians at 10^6, so it is formed in 64 bits and reduced there to the nearest quarter
//    turn; what is left, within pi / 4, goes to float32 (an error of 2^-25) and through the
//    series of sine and cosine, cut where the next term is below 2^-25.
//  * A thread holds the sines and cosines of one group of pairs (16 bytes of a row, 32 with
//    halves) of one token and goes over some heads with them, so that angles cost little
//    beside the rows.  What bounds the call is HBM, or the launch.  (16k tokens of 40 heads of 128
//    bf16 columns, 336 MB, 57 to 69 us by where its tensors lie, 4.9 to 5.9 TB/s, the kernel over one set
//    of tensors 55, 6.1; a chunk of 4096 tokens stored, 101 MB, 20.6 us, 4.9; a large copy 4.9.)
#include <type_traits>

#include "grkv_device.h"
#include "grkv_internal.h"

namespace grkv {
namespace {

constexpr int kRoTh = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// sin and cos of a turn by x: |x| <= pi / 4.  Series of both up to x^9 and x^8; the next
// terms are below 2^-28 and 2^-25.
__device__ __forceinline__ void sin_cos(float x, float* s, float* c) {
  const float z = x * x;
  *s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  *c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -.5f), 1.f);
}

// The same of any angle p f, times `scale`.
__device__ __forceinline__ void turn(int p, double f, float scale, bool inverse, float* s, float* c) {
  const double quarters = (double)p * f * 0.63661977236758134308;   // 2 / pi
  const double n = __builtin_rint(quarters);
  // (whole turns leave before the conversion, so that any finite number of them is right)
  const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  float sn, cs;
  sin_cos((float)((quarters - n) * 1.57079632679489661923), &sn, &cs);
  const float s1 = q & 1 ? cs : sn, c1 = q & 1 ? sn : cs;
  *s = (((q & 2) != 0) != inverse ? -s1 : s1) * scale;
  *c = (((q + 1) & 2) != 0 ? -c1 : c1) * scale;
}

__device__ __forceinline__ float value(u16 x) { return bf16_to_f32(x); }
__device__ __forceinline__ float value(float x) { return x; }

// N neighbouring columns as floats, by loads of 16 bytes where N fills them, which pass the
// caches: rows are read once (16k tokens of 40 heads, six tensors used in turn, 66.6 -> 56.9 us
// where those lay, 67 to 69 where others do; stored so too 57.1).
template <int N, typename T>
__device__ __forceinline__ void load_cols(const T* p, float (&x)[N]) {
  constexpr int V = 16 / sizeof(T);
  if constexpr (N % V == 0) {
#pragma unroll
    for (int k = 0; k < N; k += V) {
      const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + k));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
          x[k + 2 * i] = __uint_as_float(w[i] << 16);
          x[k + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          x[k + i] = __uint_as_float(w[i]);
        }
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = value(p[k]);
  }
}

// ... and stored, rounded to T; VEC: p is a multiple of N columns that are 8 bytes or more.
template <bool VEC, int N, typename T>
__device__ __forceinline__ void store_cols(T* p, const float (&x)[N]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 4) {
      static_assert(N % 4 == 0, "whole 16 bytes");
#pragma unroll
      for (int k = 0; k < N; k += 4)
        *reinterpret_cast<f32x4*>(p + k) = (f32x4){x[k], x[k + 1], x[k + 2], x[k + 3]};
    } else {
      static_assert(N % 4 == 0, "whole 8 bytes");
      uint32_t w[N / 2];
#pragma unroll
      for (int k = 0; k < N; k += 2)
        w[k / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[k], x[k + 1]}, bf16x2));
      if constexpr (N % 8 == 0) {
#pragma unroll
        for (int k = 0; k < N / 2; k += 4)
          *reinterpret_cast<u32x4*>(p + 2 * k) = (u32x4){w[k], w[k + 1], w[k + 2], w[k + 3]};
      } else {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if constexpr (sizeof(T) == 2) *reinterpret_cast<__bf16*>(p + k) = (__bf16)x[k];
      else p[k] = x[k];
    }
  }
}

// A head's columns in pieces, one per thread: PAIRS pairs each (with halves, that many
// columns of either), then W of the columns that are not turned.
template <typename T, bool INTER, bool VEC>
struct Pieces {
  static constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
  static constexpr int PAIRS = INTER && VEC ? V / 2 : V;
  static constexpr int W = V;
};

// Sines and cosines of the pairs of one piece at one position.
template <int PAIRS>
struct Turn {
  float s[PAIRS], c[PAIRS];
  __device__ __forceinline__ void make(const RotaryK& r, int pos, int first) {
#pragma unroll
    for (int k = 0; k < PAIRS; ++k) turn(pos, r.freqs[first + k], r.scale, r.inverse, s + k, c + k);
  }
};

// One piece of one row: turned where piece < r.turned, else copied.
template <typename T, typename TO, bool INTER, bool VEC, int PAIRS>
__device__ __forceinline__ void piece_row(const RotaryK& r, const Turn<PAIRS>& t, int piece, const T* x, TO* y) {
  using P = Pieces<T, INTER, VEC>;
  static_assert(PAIRS == P::PAIRS, "a thread's pairs");
  if (piece < r.turned) {
    const int i = piece * PAIRS;
    if constexpr (INTER) {
      float v[2 * PAIRS], w[2 * PAIRS];
      load_cols<2 * PAIRS>(x + 2 * i, v);
#pragma unroll
      for (int k = 0; k < PAIRS; ++k) {
        w[2 * k] = fmaf(v[2 * k], t.c[k], -(v[2 * k + 1] * t.s[k]));
        w[2 * k + 1] = fmaf(v[2 * k], t.s[k], v[2 * k + 1] * t.c[k]);
      }
      store_cols<VEC>(y + 2 * i, w);
    } else {
      const int half = r.dims / 2;
      float a[PAIRS], b[PAIRS], u[PAIRS], w[PAIRS];
      load_cols<PAIRS>(x + i, a);
      load_cols<PAIRS>(x + half + i, b);
#pragma unroll
      for (int k = 0; k < PAIRS; ++k) {
        u[k] = fmaf(a[k], t.c[k], -(b[k] * t.s[k]));
        w[k] = fmaf(a[k], t.s[k], b[k] * t.c[k]);
      }
      store_cols<VEC>(y + i, u);
      store_cols<VEC>(y + half + i, w);
    }
  } else {
    const int at = r.dims + (piece - r.turned) * P::W;
    float v[P::W];
    load_cols<P::W>(x + at, v);
    store_cols<VEC>(y + at, v);
  }
}

template <typename T, bool INTER, bool VEC>
__global__ __launch_bounds__(kRoTh) void rotary_kernel(RotaryK r) {
  using P = Pieces<T, INTER, VEC>;
  const uint32_t item = blockIdx.x * kRoTh + threadIdx.x;
  const uint32_t t = item / (uint32_t)r.pieces;
  if (t >= r.tokens) return;
  const int piece = (int)(item - t * r.pieces);
  const int pos = r.positions[t];
  if (pos == GRKV_NO_POSITION) return;
  Turn<P::PAIRS> tn;
  if (piece < r.turned) tn.make(r, pos, piece * P::PAIRS);
  const int h0 = blockIdx.y * r.per, h1 = min(r.heads, h0 + r.per);
  const T* x = (const T*)r.x.data + t * r.x.token_stride;
  T* y = (T*)r.y.data + t * r.y.token_stride;
#pragma unroll 4
  for (int h = h0; h < h1; ++h)
    piece_row<T, T, INTER, VEC>(r, tn, piece, x + h * r.x.head_stride, y + h * r.y.head_stride);
}

// Heads of a launch: those of q, then k, then v; a block's are of one kind.
template <typename T, typename TP, bool INTER, bool VEC>
__global__ __launch_bounds__(kRoTh) void store_kernel(StoreK a) {
  using P = Pieces<T, INTER, VEC>;
  const RotaryK& r = a.r;
  const uint32_t item = blockIdx.x * kRoTh + threadIdx.x;
  const uint32_t t = item / (uint32_t)r.pieces;
  if (t >= r.tokens) return;
  const int piece = (int)(item - t * r.pieces);
  int g = blockIdx.y;
  const bool q = g < a.q_groups;
  if (!q) g -= a.q_groups;
  const bool v = !q && g >= a.k_groups;
  if (v) g -= a.k_groups;
  const int h0 = g * r.per, h1 = min(q ? r.heads : a.heads, h0 + r.per);
  int pos = 0;
  if (r.turned > 0) {
    pos = r.positions[t];
    if (pos == GRKV_NO_POSITION) return;
  }
  Turn<P::PAIRS> tn;
  if (!v && piece < r.turned) tn.make(r, pos, piece * P::PAIRS);
  if (q) {
    const T* x = (const T*)r.x.data + t * r.x.token_stride;
    T* y = (T*)r.y.data + t * r.y.token_stride;
#pragma unroll 4
    for (int h = h0; h < h1; ++h)
      piece_row<T, T, INTER, VEC>(r, tn, piece, x + h * r.x.head_stride, y + h * r.y.head_stride);
    return;
  }
  const grkv_rows& in = v ? a.v : a.k;
  TP* pool = (TP*)(v ? a.pool_v : a.pool_k);
  const T* x = (const T*)in.data + t * in.token_stride;
  const int64_t* slots = a.slots + t * a.slot_stride;
#pragma unroll 2
  for (int h = h0; h < h1; ++h) {
    const int64_t slot = slots[h];
    if ((uint64_t)slot >= (uint64_t)a.rows) continue;   // (no row: -1)
    const T* row = x + h * in.head_stride;
    TP* to = pool + (size_t)slot * r.d;
    if (!v) {
      piece_row<T, TP, INTER, VEC>(r, tn, piece, row, to);
    } else if (piece < r.turned) {   // a piece of values: the same columns as they are
      constexpr int N = INTER ? 2 * P::PAIRS : P::PAIRS;
      float w[N];
      load_cols<N>(row + piece * N, w);
      store_cols<VEC>(to + piece * N, w);
      if constexpr (!INTER) {
        load_cols<N>(row + r.dims / 2 + piece * N, w);
        store_cols<VEC>(to + r.dims / 2 + piece * N, w);
      }
    } else {
      const int at = r.dims + (piece - r.turned) * P::W;
      float w[P::W];
      load_cols<P::W>(row + at, w);
      store_cols<VEC>(to + at, w);
    }
  }
}

bool rows_fit(const grkv_rows& r, int esize) {
  return ((uintptr_t)r.data & 15) == 0 && r.token_stride * esize % 16 == 0 && r.head_stride * esize % 16 == 0;
}

// The pieces of a head, and how many heads a thread takes: four where threads are many
// enough to fill the card (1024 SIMDs, eight waves each), else down to one.  (16k tokens of 40
// heads, 2 / 4 / 8 heads: 67.9 / 68.8 / 70.2 us.)
void plan(RotaryK* r, int esize, bool vec, int heads) {
  const int v = vec ? 16 / esize : 1, pairs = r->interleaved && vec ? v / 2 : v;
  r->turned = r->dims / 2 / pairs;
  r->pieces = r->turned + (r->d - r->dims) / v;
  r->per = 1;
  const int64_t threads = (int64_t)r->tokens * r->pieces * heads;
  while (r->per < 4 && threads / (2 * r->per) >= 1024 * 8 * 64) r->per *= 2;
}

// Whether 16 bytes are whole pairs (or columns of one half) everywhere.
bool whole(const RotaryK& r, int esize) {
  const int v = 16 / esize;
  return (r.interleaved ? r.dims : r.dims / 2) % v == 0 && (r.d - r.dims) % v == 0;
}

template <typename T>
hipError_t launch_rotary_t(RotaryK r, hipStream_t s) {
  const bool vec = whole(r, sizeof(T)) && rows_fit(r.x, sizeof(T)) && rows_fit(r.y, sizeof(T));
  plan(&r, sizeof(T), vec, r.heads);
  const dim3 grid((unsigned)(((int64_t)r.tokens * r.pieces + kRoTh - 1) / kRoTh), (r.heads + r.per - 1) / r.per);
  const dim3 th(kRoTh);
  if (r.interleaved) {
    if (vec) hipLaunchKernelGGL((rotary_kernel<T, true, true>), grid, th, 0, s, r);
    else hipLaunchKernelGGL((rotary_kernel<T, true, false>), grid, th, 0, s, r);
  } else {
    if (vec) hipLaunchKernelGGL((rotary_kernel<T, false, true>), grid, th, 0, s, r);
    else hipLaunchKernelGGL((rotary_kernel<T, false, false>), grid, th, 0, s, r);
  }
  return hipGetLastError();
}

template <typename T, typename TP>
hipError_t launch_store_t(StoreK a, hipStream_t s) {
  RotaryK& r = a.r;
  const bool vec = whole(r, sizeof(T)) && rows_fit(a.k, sizeof(T)) && rows_fit(a.v, sizeof(T)) &&
                   rows_fit(r.x, sizeof(T)) && rows_fit(r.y, sizeof(T));
  plan(&r, sizeof(T), vec, r.heads + 2 * a.heads);
  a.q_groups = (r.heads + r.per - 1) / r.per;
  a.k_groups = (a.heads + r.per - 1) / r.per;
  const dim3 grid((unsigned)(((int64_t)r.tokens * r.pieces + kRoTh - 1) / kRoTh), a.q_groups + 2 * a.k_groups);
  const dim3 th(kRoTh);
  if (r.interleaved) {
    if (vec) hipLaunchKernelGGL((store_kernel<T, TP, true, true>), grid, th, 0, s, a);
    else hipLaunchKernelGGL((store_kernel<T, TP, true, false>), grid, th, 0, s, a);
  } else {
    if (vec) hipLaunchKernelGGL((store_kernel<T, TP, false, true>), grid, th, 0, s, a);
    else hipLaunchKernelGGL((store_kernel<T, TP, false, false>), grid, th, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryK& r, int dtype, hipStream_t s) {
  return dtype == GRKV_BF16 ? launch_rotary_t<u16>(r, s) : launch_rotary_t<float>(r, s);
}

hipError_t launch_store(const StoreK& a, int dtype, int pool_dtype, hipStream_t s) {
  if (dtype == GRKV_BF16)
    return pool_dtype == GRKV_BF16 ? launch_store_t<u16, u16>(a, s) : launch_store_t<u16, float>(a, s);
  return pool_dtype == GRKV_BF16 ? launch_store_t<float, u16>(a, s) : launch_store_t<float, float>(a, s);
}

}  // namespace grkv
