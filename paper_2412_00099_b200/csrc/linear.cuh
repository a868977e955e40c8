// What the kernels of the experts' products share: the groups of rows, the activations, the 8-bit blocks, and what happens to a
// value once its sum is formed.  All of them end with a warp that holds 32 neighbouring columns of several rows: four lanes have a row's, eight each.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mcce.h"

namespace mcce {
namespace linear {

// Every kernel here is launched so that it may take its place as soon as the last CTAs of the kernel before it leave, without the time between two launches, and
// waits for that one's memory before it touches any (one token, gated: 12.3 -> 10.7 us).  None lets the next one in sooner: CTAs that only wait were in
// the way of those that work (198 rows x 259 x 515 fp32 13.5 -> 27 us).
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... P>
cudaError_t launch_close(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, const std::decay_t<P>&... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st, cfg.attrs = attr, cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

enum Kind { kForward = 0, kBackward = 1, kDweight = 2 };

// Rows sorted by group g = layer * E + expert.  Whatever the offsets hold, no row outside its layer is touched.
// They are read by plain loads: the kernel may be running while the one that writes them still is, and a load through the read-only path (__ldg, .nc)
// promises that nobody writes them while it runs, so that it might move up before the wait.
struct Groups {
  const int32_t* offsets;   // [L, E + 1]
  int32_t E, G;             // experts per layer, groups L * E
  int64_t R;                // rows per layer
};
struct GroupRows {
  int64_t first;   // row among the L * R rows
  int64_t m;
};
__device__ __forceinline__ GroupRows group_rows(const Groups& g, int i) {
  const int l = i / g.E;
  const int32_t* o = g.offsets + i + l;
  const int64_t lo = min(max((int64_t)*o, (int64_t)0), g.R);
  const int64_t hi = min(max((int64_t)o[1], lo), g.R);
  return {l * g.R + lo, hi - lo};
}

__device__ __forceinline__ float load_as_float(const float* p) { return *p; }
__device__ __forceinline__ float load_as_float(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// ---- activations: value and slope --------------------------------------------------------------------------
// silu(z) = z s(z) with s(z) = 1 / (1 + e^-z); slope s (1 + z (1 - s)).  gelu(z) = z P(z) with P the normal distribution; slope P + z p(z).
// FAST: bf16 results, whose rounding (2^-8) hides the (2 + |z|) 2^-22 of the fast exponential and division.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z) {
  if (FAST) return __fdividef(1.f, 1.f + __expf(-z));   // 0 from about z = -87 on
  return 1.f / (1.f + expf(-z));
}
// For fp32 results of bf16 rows, which hide nothing: the exponential in full; its argument's sign is chosen so that the divisor lies in 1 .. 2, where the
// short division is off by two steps at most.  8192 rows x 1024 x 4096, silu: 62 us with the fast exponential, 66 so, 76 with the full division.
__device__ __forceinline__ float sigmoid_wide(float z) {
  const float e = expf(-fabsf(z));
  return __fdividef(z < 0.f ? e : 1.f, 1.f + e);
}
template <bool FAST>
__device__ __forceinline__ void slope_and_value(float z, int act, float& value, float& slope) {
  if (act == MCCE_ACT_SILU) {
    const float s = sigmoid<FAST>(z);
    value = z * s, slope = fmaf(value, 1.f - s, s);
  } else if (act == MCCE_ACT_GELU) {
    const float p = normcdff(z), q = z * z * -0.5f;
    value = z * p, slope = p + z * (0.3989422804014327f * (FAST ? __expf(q) : expf(q)));
  } else {
    value = z, slope = 1.f;
  }
}

// ---- blocks of 32 columns in 8 bits --------------------------------------------------------------------------
// Scale byte b stands for 2^(b - 127).  The scale is the smallest power of two that brings the block's largest magnitude to 448 = 1.75 2^8 at
// most: with the largest 1.f 2^(E - 127) that is b = E - 8, one more if 1.f > 1.75.  Dividing by it is exact, so a value is rounded once.
// A block with a NaN or an infinity has scale and values NaN.
__device__ __forceinline__ uint32_t block_scale(uint32_t largest_bits) {
  const uint32_t e = largest_bits >> 23;
  if (e == 255u) return 255u;
  const int b = (int)e - 8 + ((largest_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b > 0 ? (uint32_t)b : 0u;
}
__device__ __forceinline__ float scale_inverse(uint32_t scale) { return __uint_as_float(scale == 255u ? 0x7fffffffu : (254u - scale) << 23); }
__device__ __forceinline__ float scale_value(uint32_t scale) {
  return __uint_as_float(scale == 255u ? 0x7fffffffu : scale == 0u ? 0x00400000u : scale << 23);
}
__device__ __forceinline__ uint32_t to_e4m3x2(float low, float high) {
  return __nv_cvt_float2_to_fp8x2(make_float2(low, high), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3x2_value(uint32_t pair) {
  return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
}

// The scale of the values that a whole warp holds, a column per lane; lanes without one hand in 0.
__device__ __forceinline__ uint32_t warp_block_scale(float v) {
  return block_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
}

// ---- eight neighbouring columns of a row in a lane ----------------------------------------------------------------
// As they lie in memory, `count` of them (1 .. 8; the rest reads as 0), in one or two accesses where `wide` says that they are aligned to it.
template <typename E>
__device__ __forceinline__ void load_8(const E* p, bool wide, int count, uint32_t (&w)[2 * sizeof(E)]) {
  if (wide && count == 8) {
    if constexpr (sizeof(E) == 1) {
      const uint2 v = *(const uint2*)p;
      w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i) {
        const uint4 v = ((const uint4*)p)[i];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 2 * (int)sizeof(E); ++i) w[i] = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) {
      if constexpr (sizeof(E) == 4) w[j] = __float_as_uint(p[j]);
      else if constexpr (sizeof(E) == 2) w[j / 2] |= (uint32_t)((const uint16_t*)p)[j] << (16 * (j & 1));
      else w[j / 4] |= (uint32_t)p[j] << (8 * (j & 3));
    }
}
__device__ __forceinline__ void floats_of(const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void floats_of(const uint32_t (&w)[4], float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[2 * j] = __uint_as_float(w[j] << 16), v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
}
__device__ __forceinline__ void floats_of(const uint32_t (&w)[2], float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = e4m3x2_value(w[j / 2] >> (16 * (j & 1)) & 0xffffu);
    v[2 * j] = f.x, v[2 * j + 1] = f.y;
  }
}
template <typename E>
__device__ __forceinline__ void store_words_8(E* p, bool wide, int count, const uint32_t (&w)[2 * sizeof(E)]) {
  if (wide && count == 8) {
    if constexpr (sizeof(E) == 1) {
      *(uint2*)p = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i) ((uint4*)p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) {
      if constexpr (sizeof(E) == 4) p[j] = __uint_as_float(w[j]);
      else if constexpr (sizeof(E) == 2) ((uint16_t*)p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
      else p[j] = (uint8_t)(w[j / 4] >> (8 * (j & 3)));
    }
}
__device__ __forceinline__ void store_8(float* p, bool wide, int count, const float (&v)[8]) {
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
  store_words_8(p, wide, count, w);
}
__device__ __forceinline__ void store_8(__nv_bfloat16* p, bool wide, int count, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    w[j] = *(const uint32_t*)&h;
  }
  store_words_8(p, wide, count, w);
}
// Bits of the largest magnitude, ordered like the magnitudes, infinity and NaN last
__device__ __forceinline__ uint32_t largest_bits(const float (&v)[8]) {
  uint32_t bits = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) bits = max(bits, __float_as_uint(v[j]) & 0x7fffffffu);
  return bits;
}
__device__ __forceinline__ uint32_t largest_bits(const uint32_t (&w)[8]) {
  uint32_t bits = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) bits = max(bits, w[j] & 0x7fffffffu);
  return bits;
}
__device__ __forceinline__ uint32_t largest_bits(const uint32_t (&w)[4]) {   // bf16, two at a time
  __nv_bfloat162 m = __habs2(*(const __nv_bfloat162*)&w[0]);
#pragma unroll
  for (int j = 1; j < 4; ++j) m = __hmax2_nan(m, __habs2(*(const __nv_bfloat162*)&w[j]));
  const uint32_t b = *(const uint32_t*)&m;
  return max(b << 16, b & 0xffff0000u);
}
// The same in 8 bits, and the scale of the 32 columns that this lane and its three neighbours hold, `bits` being this lane's largest; values behind the last
// column are 0.  Every lane of the warp calls it.
__device__ __forceinline__ uint32_t pack_8(const float (&v)[8], uint32_t bits, uint32_t (&w)[2]) {
  bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
  bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
  const uint32_t s = block_scale(bits);
  const float f = scale_inverse(s);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = to_e4m3x2(v[4 * i] * f, v[4 * i + 1] * f) | to_e4m3x2(v[4 * i + 2] * f, v[4 * i + 3] * f) << 16;
  return s;
}

// ---- what becomes of a sum -----------------------------------------------------------------------------------
struct ForwardArgs {
  const void *bias, *bias_up;   // [G, n], fp32 or T; may be null
  const void* add;              // like out; may be null, may be out
  void* out;
  void* saved;                  // [rows, n (2 n gated)] T or e4m3, or null
  uint8_t* scales;              // [rows, blocks (2 blocks gated)] with e4m3
  int64_t ld_add, ld_out, ld_saved;
  int32_t bias_f32, out_f32, act, n, blocks;
  int32_t wide;                 // eight columns of every tensor's rows are aligned as a whole (16 bytes at most)
};
struct BackwardArgs {
  const void *add, *saved;      // saved: [rows, k (2 k below == 2)] T or e4m3
  const uint8_t* scales;
  void *dx, *h;
  int64_t ld_add, ld_saved, ld_dx, ld_h;
  int32_t below, act, k, blocks, wide;   // below: 0 none, 1 an activation, 2 a gated one
};

// P times eight rows from `row` on, of which the first `left` count: lane l has rows l / 4, 8 + l / 4 .., columns f .. f + 7 with f the tile's
// first + 8 (l % 4): z, and z_up of a gated layer.  A warp calls it as a whole, with the same rows.  (With a column per lane and a row after the other the
// gradient through a gated layer took five times as many instructions.)  What is read is read without a condition (behind the last row that counts, that
// row again: a branch around every load made the loads wait for one another).
template <typename T, bool GATED>
struct Forward {
  const ForwardArgs& a;
  float b[8] = {}, b_up[8] = {};
  int f, count;   // columns that exist
  __device__ __forceinline__ void bias_of(const void* p, int64_t at, float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) v[j] = a.bias_f32 ? ((const float*)p)[at + j] : load_as_float((const T*)p + at + j);
  }
  __device__ __forceinline__ Forward(const ForwardArgs& a_, int group, int f_) : a(a_), f(f_), count(min(max(a_.n - f_, 0), 8)) {
    if (!a.bias) return;
    bias_of(a.bias, (int64_t)group * a.n + f, b);
    if (GATED) bias_of(a.bias_up, (int64_t)group * a.n + f, b_up);
  }
  __device__ __forceinline__ void keep(int64_t row, bool on, const float (&v)[8], int half) const {
    if (a.scales) {
      float z[8];
      uint32_t w[2];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = j < count ? v[j] : 0.f;
      const uint32_t s = pack_8(z, largest_bits(z), w);
      if (!on || count == 0) return;
      store_words_8((uint8_t*)a.saved + row * a.ld_saved + half * a.n + f, a.wide && (!half || a.n % 8 == 0), count, w);
      if ((f & 31) == 0) a.scales[row * (GATED ? 2 * a.blocks : a.blocks) + half * a.blocks + (f >> 5)] = (uint8_t)s;
    } else if (on && count) {
      store_8((T*)a.saved + row * a.ld_saved + half * a.n + f, a.wide && (!half || a.n % 8 == 0), count, v);
    }
  }
  template <typename O, int P>
  __device__ __forceinline__ void finish(int64_t row, int left, float (&z)[P][8], float (&up)[P][8]) const {
    constexpr bool kFast = sizeof(O) == 2, kWide = sizeof(T) == 2 && sizeof(O) == 4;
    const int r = (threadIdx.x & 31) >> 2;
    uint32_t add[P][2 * sizeof(O)] = {};
    if (a.add && count) {
#pragma unroll
      for (int i = 0; i < P; ++i) load_8((const O*)a.add + (row + min(r + 8 * i, left - 1)) * a.ld_add + f, a.wide, count, add[i]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[i][j] += b[j];
        if (GATED) up[i][j] += b_up[j];
      }
    if (a.saved) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        keep(row + r + 8 * i, r + 8 * i < left, z[i], 0);
        if (GATED) keep(row + r + 8 * i, r + 8 * i < left, up[i], 1);
      }
    }
    if (a.act == MCCE_ACT_SILU) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] *= kWide ? sigmoid_wide(z[i][j]) : sigmoid<kFast>(z[i][j]);
    } else if (a.act == MCCE_ACT_GELU) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] *= normcdff(z[i][j]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float y[8];
      floats_of(add[i], y);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] += GATED ? z[i][j] * up[i][j] : z[i][j];
      if (r + 8 * i < left && count) store_8((O*)a.out + (row + r + 8 * i) * a.ld_out + f, a.wide, count, y);
    }
  }
  template <int P>
  __device__ __forceinline__ void rows(int64_t row, int left, float (&z)[P][8], float (&up)[P][8]) const {
    if (left <= 0) return;
    if (a.out_f32) finish<float, P>(row, left, z, up);
    else finish<T, P>(row, left, z, up);
  }
};

// The same for a gradient with respect to rows, t, in two steps: `ask` reads what the layer below kept (or what is added), `rows` uses it, so
// that a caller can wait for its sums in between.
template <typename T>
struct Backward {
  const BackwardArgs& a;
  int f, count;
  bool wide_up;   // the second half of the columns too
  __device__ __forceinline__ Backward(const BackwardArgs& a_, int, int f_)
      : a(a_), f(f_), count(min(max(a_.k - f_, 0), 8)), wide_up(a_.wide && a_.k % 8 == 0) {}
  template <int P>
  struct Asked {
    uint32_t z[P][2 * sizeof(T)], up[P][2 * sizeof(T)], scales[P];   // as they lie in memory; scales: z's in the low byte, up's in the next
  };
  template <int P>
  __device__ __forceinline__ void ask(int64_t row, int left, Asked<P>& q) const {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      q.scales[i] = 0u;
#pragma unroll
      for (int j = 0; j < 2 * (int)sizeof(T); ++j) q.z[i][j] = q.up[i][j] = 0u;
    }
    if (!count || left <= 0) return;
    const int r = (threadIdx.x & 31) >> 2;
    if (a.below && a.scales) {
      uint32_t su[P] = {};
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int64_t at = row + min(r + 8 * i, left - 1);
        const uint8_t *p = (const uint8_t*)a.saved + at * a.ld_saved + f, *s = a.scales + at * a.below * a.blocks + (f >> 5);
        uint32_t w[2];
        load_8(p, a.wide, count, w);
        q.z[i][0] = w[0], q.z[i][1] = w[1], q.scales[i] = s[0];
        if (a.below == 2) {
          load_8(p + a.k, wide_up, count, w);
          q.up[i][0] = w[0], q.up[i][1] = w[1], su[i] = s[a.blocks];
        }
      }
#pragma unroll
      for (int i = 0; i < P; ++i) q.scales[i] |= su[i] << 8;
    } else if (a.below || a.add) {
      const T* p = (const T*)(a.below ? a.saved : a.add) + f;
      const int64_t ld = a.below ? a.ld_saved : a.ld_add;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const T* at = p + (row + min(r + 8 * i, left - 1)) * ld;
        load_8(at, a.wide, count, q.z[i]);
        if (a.below == 2) load_8(at + a.k, wide_up, count, q.up[i]);
      }
    }
  }
  template <int P>
  __device__ __forceinline__ void rows(int64_t row, int left, const float (&t)[P][8], const Asked<P>& q) const {
    if (!count || left <= 0) return;
    const int r = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const bool on = r + 8 * i < left;
      T* dx = (T*)a.dx + (row + r + 8 * i) * a.ld_dx + f;
      float z[8], up[8], slope[8], v[8];
      if (a.below && a.scales) {
        const uint32_t wz[2] = {q.z[i][0], q.z[i][1]}, wu[2] = {q.up[i][0], q.up[i][1]};
        const float sz = scale_value(q.scales[i] & 255u), su = scale_value(q.scales[i] >> 8);
        floats_of(wz, z), floats_of(wu, up);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] *= sz, up[j] *= su;
      } else {
        floats_of(q.z[i], z), floats_of(q.up[i], up);
      }
      if (!a.below) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t[i][j] + z[j];
        if (on) store_8(dx, a.wide, count, v);
        continue;
      }
      if (a.act == MCCE_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) slope_and_value<sizeof(T) == 2>(z[j], MCCE_ACT_SILU, z[j], slope[j]);
      } else if (a.act == MCCE_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) slope_and_value<sizeof(T) == 2>(z[j], MCCE_ACT_GELU, z[j], slope[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) slope[j] = 1.f;
      }
      T* h = (T*)a.h + (row + r + 8 * i) * a.ld_h + f;
      if (a.below == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t[i][j] * up[j] * slope[j];
        if (on) store_8(dx, a.wide, count, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t[i][j] * z[j];
        if (on) store_8(dx + a.k, wide_up, count, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = z[j] * up[j];
        if (on && a.h) store_8(h, a.wide, count, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t[i][j] * slope[j];
        if (on) store_8(dx, a.wide, count, v);
        if (on && a.h) store_8(h, a.wide, count, z);
      }
    }
  }
};

// ---- one call ---------------------------------------------------------------------------------------------------
struct Problem {
  Groups groups;
  int32_t n, k, gated;             // sizes of the weights [n, k]; two of them when gated
  int64_t L, ld_x, ld_y, ld_w, step_w, half_y;   // y: dout (the gradients), its second half half_y columns on
  const void *x, *y, *w, *w_up;    // forward: x, w; backward: y, w; dweight: y, x
  void *dw, *dw_up;                // dweight
  const void *add_dw, *add_dw_up;
  int32_t dw_f32, dw_wide;   // dw_wide: of its rows (and of those added) four columns (1), also 16 bytes (2), are aligned as a whole
  ForwardArgs fwd;
  BackwardArgs bwd;
};

// Tile number -> (group, tile of rows) through the running number of tiles before every group, in shared memory.
__device__ __forceinline__ int find_group(const int* before, int G, int tile) {
  int lo = 0, hi = G;   // before[lo] <= tile < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= tile) lo = mid;
    else hi = mid;
  }
  return lo;
}
// before[0 .. G]: every thread of the block calls it; ends with a barrier.  scratch: 33 ints.
__device__ __forceinline__ void count_tiles(const Groups& g, int rows_per_tile, int* before, int* scratch) {
  const int t = threadIdx.x, nt = blockDim.x, each = (g.G + nt - 1) / nt;
  auto tiles = [&](int i) { return (int)((group_rows(g, i).m + rows_per_tile - 1) / rows_per_tile); };
  int sum = 0;
  for (int i = t * each; i < min((t + 1) * each, g.G); ++i) sum += tiles(i);
  int run = sum;
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, run, d);
    if ((t & 31) >= d) run += o;
  }
  if ((t & 31) == 31) scratch[t >> 5] = run;
  __syncthreads();
  // tiles of the warps before this one, and of all
  int w = (t & 31) < (nt >> 5) ? scratch[t & 31] : 0, all = w, less = (t & 31) < (t >> 5) ? w : 0;
  all = __reduce_add_sync(0xffffffffu, all), less = __reduce_add_sync(0xffffffffu, less);
  run += less - sum;
  if (t == 0) before[g.G] = all;
  if (each == 1) {
    if (t < g.G) before[t] = run;
  } else {
    for (int i = t * each; i < min((t + 1) * each, g.G); ++i) before[i] = run, run += tiles(i);
  }
  __syncthreads();
}

cudaError_t run_general(Kind kind, const Problem& p, int32_t dtype, cudaStream_t st);   // any size, stride and alignment
bool few_applicable(const Problem& p, int32_t dtype);   // forward, a few rows in all
cudaError_t run_few(const Problem& p, cudaStream_t st);
bool tensor_applicable(Kind kind, const Problem& p, int32_t dtype);
cudaError_t run_tensor(Kind kind, const Problem& p, cudaStream_t st);
int bias_chunks(int64_t rows, int32_t G, int32_t n);   // more than one: run_bias_sums needs `parts`
cudaError_t run_bias_sums(const Problem& p, int32_t dtype, const void* add, const void* add_up, void* db, void* db_up, float* parts,
                          cudaStream_t st);
cudaError_t run_align(const void* from, int64_t rows, int64_t per, int32_t cols, int64_t ld, int64_t step, void* to, int64_t ld_to, cudaStream_t st);
cudaError_t run_pack(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, uint8_t* q, uint8_t* scales,
                     cudaStream_t st);
cudaError_t run_unpack(const uint8_t* q, const uint8_t* scales, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, void* x,
                       cudaStream_t st);

}  // namespace linear
}  // namespace mcce
