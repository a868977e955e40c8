// U consecutive columns of a row as one load or store, for the row operators (norm.cu, rows.cu): U is 8, 4, 2 or 1,
// the widest that the width, the strides and the addresses of a call allow.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace mcce {

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

// The U values as they lie in memory: one 16-byte vector at most, eight fp32 are two of them.
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
  __device__ __forceinline__ void get(float (&v)[U]) const {
    const T* e = (const T*)r;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if constexpr (sizeof(T) == 2) v[i] = __bfloat162float(e[i]);
      else v[i] = e[i];
    }
  }
  // round to nearest even, once
  __device__ __forceinline__ void set(const float (&v)[U]) {
    T* e = (T*)r;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if constexpr (sizeof(T) == 2) e[i] = __float2bfloat16_rn(v[i]);
      else e[i] = v[i];
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = Raw{};
  }
};

// Host: the widest unit that divides d and for which every row of every tensor starts aligned.
struct UnitRule {
  int u;
  explicit UnitRule(int d) : u(d % 8 == 0 ? 8 : d % 4 == 0 ? 4 : d % 2 == 0 ? 2 : 1) {}
  void tensor(const void* p, int64_t ld, int elem_bytes) {   // null: not part of the call
    while (p && u > 1) {
      const int a = u * elem_bytes > 16 ? 16 : u * elem_bytes;
      if ((uintptr_t)p % a == 0 && (ld * elem_bytes) % a == 0) return;
      u /= 2;
    }
  }
};

}  // namespace mcce
