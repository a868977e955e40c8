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
  __device__ __forceinline__ void get(float (&v)[U]) const {
    T e[U];
    memcpy(e, r, sizeof(e));
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = wide(e[i]);
  }
  __device__ __forceinline__ void get(float2 (&v)[U / 2]) const {
    if constexpr (sizeof(T) == 2) {
      uint32_t e[U / 2];
      memcpy(e, r, sizeof(e));
#pragma unroll
      for (int i = 0; i < U / 2; ++i) v[i] = make_float2(__uint_as_float(e[i] << 16), __uint_as_float(e[i] & 0xffff0000u));
    } else {
      memcpy(v, r, sizeof(v));
    }
  }
  __device__ __forceinline__ void set(const float (&v)[U]) {   // each value rounded once, to nearest even
    if constexpr (sizeof(T) == 2 && U > 1) {
      __nv_bfloat162 e[U / 2];
#pragma unroll
      for (int i = 0; i < U / 2; ++i) e[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      memcpy(r, e, sizeof(e));
    } else {
      T e[U];
#pragma unroll
      for (int i = 0; i < U; ++i) e[i] = narrow<T>(v[i]);
      memcpy(r, e, sizeof(e));
    }
  }
  __device__ __forceinline__ void set(const float2 (&v)[U / 2]) {
    if constexpr (sizeof(T) == 2) {
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

// U consecutive elements at any element's address: the aligned vectors around them, shifted into place.  Reads nothing
// outside [base, end), which the elements must lie in; vectors that would are replaced by single elements.
template <typename T, int U>
__device__ __forceinline__ void load_anywhere(Pack<T, U>& out, const T* p, const T* base, const T* end) {
  constexpr int N = U * (int)sizeof(T) / 16;
  static_assert(N >= 1, "whole vectors");
  const uintptr_t at = (uintptr_t)p;
  const int m = (int)(at & 15);
  const uint4* v = (const uint4*)(at - m);
  if ((const char*)v < (const char*)base || (const char*)(v + N + (m != 0)) > (const char*)end) {
    out.load_part(p, 0, U);
    return;
  }
  uint32_t w[4 * N + 4];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint4 q = v[i];
    w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
  }
  const uint4 q = m ? v[N] : make_uint4(0, 0, 0, 0);
  w[4 * N] = q.x, w[4 * N + 1] = q.y, w[4 * N + 2] = q.z, w[4 * N + 3] = q.w;
  if (m & 4) {
#pragma unroll
    for (int i = 0; i < 4 * N + 3; ++i) w[i] = w[i + 1];
  }
  if (m & 8) {
#pragma unroll
    for (int i = 0; i < 4 * N + 2; ++i) w[i] = w[i + 2];
  }
  uint32_t o[4 * N];
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) o[i] = __funnelshift_r(w[i], w[i + 1], (m & 3) * 8);
  memcpy(out.r, o, sizeof(o));
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
