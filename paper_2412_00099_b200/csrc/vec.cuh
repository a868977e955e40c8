// Rows read and written 16 bytes at a time, for the row operators (norm.cu, rows.cu).
//
// A unit is U = 16 / sizeof(T) consecutive elements of a row.  Three ways to lay units over a row:
//   aligned  every row of every tensor starts on a unit boundary and the width is a multiple of U;
//   ragged   any width: units follow the alignment of the row in memory, so a row may begin and end inside a unit.
//            These two units are moved element by element, all others 16 bytes at a time;
//   scalar   U = 1, for tensors whose rows are not aligned alike.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>
#include <string.h>

#include "span.h"

namespace mcce {

enum Layout3 { kAligned = 0, kRagged = 1, kScalar = 2 };

template <int BYTES>
struct RawOf;
template <>
struct RawOf<16> { using type = uint4; };
template <>
struct RawOf<8> { using type = uint2; };
template <>
struct RawOf<4> { using type = uint32_t; };
template <>
struct RawOf<2> { using type = uint16_t; };
template <>
struct RawOf<1> { using type = uint8_t; };

template <typename T>
__device__ __forceinline__ float wide(T v) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(v);
  else return v;
}
template <typename T>
__device__ __forceinline__ T narrow(float v) {   // to nearest even
  if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v);
  else return v;
}

// Two fp32 operations per instruction (each rounded to nearest even like the single one).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// U values as they lie in memory: vectors of at most 16 bytes (eight fp32 are two of them).
template <typename T, int U>
struct Pack {
  static constexpr int kBytes = U * (int)sizeof(T);
  static constexpr int kRaw = kBytes > 16 ? 16 : kBytes, kN = kBytes / kRaw;
  using Raw = typename RawOf<kRaw>::type;
  Raw r[kN];

  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = *((const Raw*)p + i);
  }
  __device__ __forceinline__ void load_const(const T* p) {   // data that no thread of the launch writes
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = __ldg((const Raw*)p + i);
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) *((Raw*)p + i) = r[i];
  }
  // elements [lo, hi) only, p is the address of element 0; the others read as zero
  __device__ __forceinline__ void load_part(const T* p, int lo, int hi) {
    T e[U];
#pragma unroll
    for (int i = 0; i < U; ++i) e[i] = i >= lo && i < hi ? p[i] : narrow<T>(0.f);
    memcpy(r, e, sizeof(e));
  }
  __device__ __forceinline__ void store_part(T* p, int lo, int hi) const {
    T e[U];
    memcpy(e, r, sizeof(e));
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i >= lo && i < hi) p[i] = e[i];
  }
  // in pairs; a single value has a zero beside it
  __device__ __forceinline__ void get(float2 (&v)[(U + 1) / 2]) const {
    if constexpr (U == 1) {
      T e;
      memcpy(&e, r, sizeof(e));
      v[0] = make_float2(wide(e), 0.f);
    } else if constexpr (sizeof(T) == 2) {
      uint32_t e[U / 2];
      memcpy(e, r, sizeof(e));
#pragma unroll
      for (int i = 0; i < U / 2; ++i) v[i] = make_float2(__uint_as_float(e[i] << 16), __uint_as_float(e[i] & 0xffff0000u));
    } else {
      memcpy(v, r, sizeof(v));
    }
  }
  // each value rounded once, to nearest even
  __device__ __forceinline__ void set(const float2 (&v)[(U + 1) / 2]) {
    if constexpr (U == 1) {
      const T e = narrow<T>(v[0].x);
      memcpy(r, &e, sizeof(e));
    } else if constexpr (sizeof(T) == 2) {
      __nv_bfloat162 e[U / 2];
#pragma unroll
      for (int i = 0; i < U / 2; ++i) e[i] = __floats2bfloat162_rn(v[i].x, v[i].y);
      memcpy(r, e, sizeof(e));
    } else {
      memcpy(r, v, sizeof(v));
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = Raw{};
  }
};

// Units of a row whose first one lies at any element's address: the aligned vectors around a unit, shifted into place.
// The shift is the same for every unit of the row, so the words to skip are a compile-time number, chosen once per row.
//   with_shift(first, n, base, end, f) calls f(how), and load_shifted<how> loads a unit; [base, end) is the tensor, outside of
//   which nothing is read (a row at its edge is read element by element), n the elements of the row from `first` on.
constexpr int kElements = -2, kInPlace = -1;   // else: whole words to skip, 0 .. 3

template <typename T, int U, int HOW>
__device__ __forceinline__ void load_shifted(Pack<T, U>& out, const T* p) {
  constexpr int N = U * (int)sizeof(T) / 16;
  static_assert(N >= 1, "whole vectors");
  if constexpr (HOW == kElements) {
    out.load_part(p, 0, U);
  } else if constexpr (HOW == kInPlace) {
    out.load(p);
  } else {
    const uint4* v = (const uint4*)((uintptr_t)p & ~(uintptr_t)15);
    uint32_t w[4 * N + 4];
#pragma unroll
    for (int i = 0; i <= N; ++i) {
      const uint4 q = v[i];
      w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
    }
    uint32_t o[4 * N];
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      if constexpr (sizeof(T) == 4) o[i] = w[HOW + i];
      else o[i] = __funnelshift_r(w[HOW + i], w[HOW + i + 1], ((uintptr_t)p & 3) * 8);
    }
    memcpy(out.r, o, sizeof(o));
  }
}

template <int V>
struct Int {
  static constexpr int value = V;
};
template <typename T, typename F>
__device__ __forceinline__ void with_shift(const T* first, int n, const T* base, const T* end, F f) {
  const uintptr_t at = (uintptr_t)first, lo = at & ~(uintptr_t)15, hi = ((uintptr_t)(first + n) + 15) & ~(uintptr_t)15;
  const int m = (int)(at & 15);
  if (m == 0) f(Int<kInPlace>{});
  else if (lo < (uintptr_t)base || hi > (uintptr_t)end) f(Int<kElements>{});
  else if (m < 4) f(Int<0>{});
  else if (m < 8) f(Int<1>{});
  else if (m < 12) f(Int<2>{});
  else f(Int<3>{});
}

// Host: which layout the tensors of a call allow.  `unit` is U; add every tensor (null: not part of the call).
struct LayoutRule {
  int d, unit, off = -1, step = -1;
  bool aligned, ragged = true;
  LayoutRule(int d_, int unit_) : d(d_), unit(unit_), aligned(d_ % unit_ == 0) {}
  void tensor(const void* p, int64_t ld, int elem_bytes) {
    if (!p) return;
    const int v = unit * elem_bytes > 16 ? 16 : unit * elem_bytes;
    if ((uintptr_t)p % v || (ld * elem_bytes) % v) aligned = false;
    const int o = (int)((uintptr_t)p / elem_bytes % unit), s = (int)(ld % unit);
    if (off < 0) off = o, step = s;
    if (o != off || s != step) ragged = false;
  }
  Layout3 layout() const { return aligned ? kAligned : ragged ? kRagged : kScalar; }
};

}  // namespace mcce
