// What the kernels of the experts' products share: the groups of rows, the activations, the 8-bit blocks, and what happens to a
// value once its sum is formed.  All of them end with a warp that holds 32 neighbouring columns of one row, a column per lane.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mcce.h"

namespace mcce {
namespace linear {

enum Kind { kForward = 0, kBackward = 1, kDweight = 2 };

// Rows sorted by group g = layer * E + expert.  Whatever the offsets hold, no row outside its layer is touched.
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
  const int64_t lo = min(max((int64_t)__ldg(o), (int64_t)0), g.R);
  const int64_t hi = min(max((int64_t)__ldg(o + 1), lo), g.R);
  return {l * g.R + lo, hi - lo};
}

__device__ __forceinline__ float load_as_float(const float* p) { return *p; }
__device__ __forceinline__ float load_as_float(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// ---- activations: value and slope --------------------------------------------------------------------------
// silu(z) = z s(z) with s(z) = 1 / (1 + e^-z); slope s (1 + z (1 - s)).  gelu(z) = z P(z) with P the normal distribution; slope P + z p(z).
// FAST: bf16 results, whose rounding (2^-9) hides the few 2^-22 of the fast exponential and division.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z) {
  if (FAST) return __fdividef(1.f, 1.f + __expf(-fmaxf(z, -80.f)));
  return 1.f / (1.f + expf(-z));
}
template <bool FAST>
__device__ __forceinline__ void slope_and_value(float z, int act, float& value, float& slope) {
  if (act == MCCE_ACT_SILU) {
    const float s = sigmoid<FAST>(z);
    value = z * s, slope = s * (1.f + z * (1.f - s));
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
// Two quotients by their scales: e4m3 in the low and the high byte
__device__ __forceinline__ uint32_t to_e4m3x2(float low, float high) {
  return __nv_cvt_float2_to_fp8x2(make_float2(low, high), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3x2_value(uint32_t low, uint32_t high) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(low | high << 8), __NV_E4M3);
  return __half22float2(__half2(h));
}
// The scale of the values that a whole warp holds, a column per lane; lanes without one hand in 0.
__device__ __forceinline__ uint32_t warp_block_scale(float v) {
  return block_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
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
};
struct BackwardArgs {
  const void *add, *saved;      // saved: [rows, k (2 k below == 2)] T or e4m3
  const uint8_t* scales;
  void *dx, *h;
  int64_t ld_add, ld_saved, ld_dx, ld_h;
  int32_t below, act, k, blocks;   // below: 0 none, 1 an activation, 2 a gated one
};

// N rows from `row` on, of which `left` count, in column f of this lane: z, and z_up of a gated layer.  A warp calls it as a whole; the N rows'
// loads, sums and stores are independent of one another, so that none waits for the row before it.
template <typename T, bool GATED>
struct Forward {
  const ForwardArgs& a;
  float b = 0.f, b_up = 0.f;
  int f;
  bool on;
  __device__ __forceinline__ Forward(const ForwardArgs& a_, int group, int f_) : a(a_), f(f_), on(f_ < a_.n) {
    if (a.bias && on) {
      const int64_t i = (int64_t)group * a.n + f;
      b = a.bias_f32 ? ((const float*)a.bias)[i] : load_as_float((const T*)a.bias + i);
      if (GATED) b_up = a.bias_f32 ? ((const float*)a.bias_up)[i] : load_as_float((const T*)a.bias_up + i);
    }
  }
  template <int N>
  __device__ __forceinline__ void keep8(int64_t row, int left, const float (&z)[N], int half) const {
    uint32_t s[N], mine = 0u;
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = warp_block_scale(on ? z[j] : 0.f);
    uint8_t* q = (uint8_t*)a.saved + row * a.ld_saved + half * a.n + f;
    uint32_t bytes[(N + 1) / 2];
#pragma unroll
    for (int j = 0; j < N; j += 2)
      bytes[j / 2] = to_e4m3x2(z[j] * scale_inverse(s[j]), j + 1 < N ? z[j + 1 < N ? j + 1 : j] * scale_inverse(s[j + 1 < N ? j + 1 : j]) : 0.f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (on && j < left) q[j * a.ld_saved] = (uint8_t)(bytes[j / 2] >> (8 * (j & 1)));
      if (j == (f & 31)) mine = s[j];
    }
    // lane j has row j's scale
    const int first = f & ~31, stride = GATED ? 2 * a.blocks : a.blocks, j = f & 31;
    if (first < a.n && j < N && j < left) a.scales[(row + j) * stride + half * a.blocks + (first >> 5)] = (uint8_t)mine;
  }
  template <int N>
  __device__ __forceinline__ void keep(int64_t row, int left, const float (&z)[N], int half) const {
    if (a.scales) return keep8(row, left, z, half);
    T* o = (T*)a.saved + row * a.ld_saved + half * a.n + f;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (on && j < left) store_as(o + j * a.ld_saved, z[j]);
  }
  template <int N, typename O>
  __device__ __forceinline__ void finish(int64_t row, int left, float (&z)[N], float (&up)[N]) const {
    constexpr bool kFast = sizeof(T) == 2;
    float add[N] = {};
    if (a.add) {
      const O* p = (const O*)a.add + row * a.ld_add + f;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (on && j < left) add[j] = load_as_float(p + j * a.ld_add);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      z[j] += b;
      if (GATED) up[j] += b_up;
    }
    if (a.saved) {
      keep(row, left, z, 0);
      if (GATED) keep(row, left, up, 1);
    }
    if (a.act == MCCE_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] *= sigmoid<kFast>(z[j]);
    } else if (a.act == MCCE_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] *= normcdff(z[j]);
    }
    O* o = (O*)a.out + row * a.ld_out + f;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (on && j < left) store_as(o + j * a.ld_out, (GATED ? z[j] * up[j] : z[j]) + add[j]);
  }
  template <int N>
  __device__ __forceinline__ void rows(int64_t row, int left, float (&z)[N], float (&up)[N]) const {
    if (a.out_f32) finish<N, float>(row, left, z, up);
    else finish<N, T>(row, left, z, up);
  }
};

// The same for a gradient with respect to rows, t[N], in two steps: `ask` reads what the layer below kept (or what is added),
// `rows` uses it, so that a caller can wait for its sums in between.
template <typename T>
struct Backward {
  const BackwardArgs& a;
  int f;
  bool on;
  __device__ __forceinline__ Backward(const BackwardArgs& a_, int, int f_) : a(a_), f(f_), on(f_ < a_.k) {}
  template <int N>
  struct Asked {
    uint32_t z[N], up[N], scales[N];   // as they lie in memory; scales: z's in the low byte, up's in the next
  };
  __device__ __forceinline__ uint32_t raw(const float* p) const { return __float_as_uint(*p); }
  __device__ __forceinline__ uint32_t raw(const __nv_bfloat16* p) const { return *(const uint16_t*)p; }
  __device__ __forceinline__ float value(uint32_t v) const { return __uint_as_float(sizeof(T) == 2 ? v << 16 : v); }
  template <int N>
  __device__ __forceinline__ void ask(int64_t row, int left, Asked<N>& q) const {
#pragma unroll
    for (int j = 0; j < N; ++j) q.z[j] = q.up[j] = q.scales[j] = 0u;
    if (!on) return;
    if (a.below && a.scales) {
      const uint8_t *p = (const uint8_t*)a.saved + row * a.ld_saved + f, *s = a.scales + row * a.below * a.blocks + (f >> 5);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) q.z[j] = p[j * a.ld_saved], q.scales[j] = s[j * a.below * a.blocks];
      if (a.below == 2) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < left) q.up[j] = p[j * a.ld_saved + a.k], q.scales[j] |= (uint32_t)s[j * 2 * a.blocks + a.blocks] << 8;
      }
    } else if (a.below) {
      const T* p = (const T*)a.saved + row * a.ld_saved + f;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) q.z[j] = raw(p + j * a.ld_saved);
      if (a.below == 2) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < left) q.up[j] = raw(p + j * a.ld_saved + a.k);
      }
    } else if (a.add) {
      const T* p = (const T*)a.add + row * a.ld_add + f;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) q.z[j] = raw(p + j * a.ld_add);
    }
  }
  template <int N>
  __device__ __forceinline__ void rows(int64_t row, int left, const float (&t)[N], const Asked<N>& q) const {
    if (!on) return;
    T* dx = (T*)a.dx + row * a.ld_dx + f;
    float z[N], up[N];
    if (a.below && a.scales) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 v = e4m3x2_value(q.z[j], q.up[j]);
        z[j] = v.x * scale_value(q.scales[j] & 255u), up[j] = v.y * scale_value(q.scales[j] >> 8);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) z[j] = value(q.z[j]), up[j] = value(q.up[j]);
    }
    if (!a.below) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) store_as(dx + j * a.ld_dx, t[j] + z[j]);
      return;
    }
    float slope[N];
    if (a.act == MCCE_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < N; ++j) slope_and_value<sizeof(T) == 2>(z[j], MCCE_ACT_SILU, z[j], slope[j]);
    } else if (a.act == MCCE_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < N; ++j) slope_and_value<sizeof(T) == 2>(z[j], MCCE_ACT_GELU, z[j], slope[j]);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) slope[j] = 1.f;
    }
    T* h = (T*)a.h + row * a.ld_h + f;
    if (a.below == 2) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) {
          store_as(dx + j * a.ld_dx, t[j] * up[j] * slope[j]);
          store_as(dx + j * a.ld_dx + a.k, t[j] * z[j]);
        }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (a.h && j < left) store_as(h + j * a.ld_h, z[j] * up[j]);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) store_as(dx + j * a.ld_dx, t[j] * slope[j]);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (a.h && j < left) store_as(h + j * a.ld_h, z[j]);
    }
  }
};

// ---- one call ---------------------------------------------------------------------------------------------------
struct Problem {
  Groups groups;
  int32_t n, k, gated;             // sizes of the weights [n, k]; two of them when gated
  int64_t L, ld_x, ld_y, ld_w, step_w;   // y: out (forward), dout (the gradients)
  const void *x, *y, *w, *w_up;    // forward: x, w; backward: y, w; dweight: y, x
  void *dw, *dw_up;                // dweight
  const void *add_dw, *add_dw_up;
  int32_t dw_f32, dw_wide;   // dw_wide: its rows (and those added) start at multiples of 16 bytes
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
  int sum = 0;
  for (int i = t * each; i < min((t + 1) * each, g.G); ++i) sum += (int)((group_rows(g, i).m + rows_per_tile - 1) / rows_per_tile);
  int run = sum;
  for (int d = 1; d < 32; d *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, run, d);
    if ((t & 31) >= d) run += o;
  }
  if ((t & 31) == 31) scratch[t >> 5] = run;
  __syncthreads();
  if (t < 32) {
    int w = t < (nt >> 5) ? scratch[t] : 0;
    for (int d = 1; d < 32; d *= 2) {
      const int o = __shfl_up_sync(0xffffffffu, w, d);
      if (t >= d) w += o;
    }
    scratch[t] = w;
  }
  __syncthreads();
  run += (t >> 5 ? scratch[(t >> 5) - 1] : 0) - sum;   // tiles before this thread's groups
  if (t == 0) before[g.G] = scratch[(nt >> 5) - 1];
  for (int i = t * each; i < min((t + 1) * each, g.G); ++i) {
    before[i] = run;
    run += (int)((group_rows(g, i).m + rows_per_tile - 1) / rows_per_tile);
  }
  __syncthreads();
}

cudaError_t run_general(Kind kind, const Problem& p, int32_t dtype, cudaStream_t st);   // any size, stride and alignment
bool tensor_applicable(Kind kind, const Problem& p, int32_t dtype);
cudaError_t run_tensor(Kind kind, const Problem& p, cudaStream_t st);
cudaError_t run_bias_sums(const Problem& p, int32_t dtype, const void* add, const void* add_up, void* db, void* db_up, cudaStream_t st);
cudaError_t run_pack(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, uint8_t* q, uint8_t* scales,
                     cudaStream_t st);
cudaError_t run_unpack(const uint8_t* q, const uint8_t* scales, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, void* x,
                       cudaStream_t st);

}  // namespace linear
}  // namespace mcce
