// The forward product for few rows (a token or a few): every touched expert's weights are read once, each row of them by a warp, for up to four rows
// of x at a time.  Nothing else costs: with one row per expert this is 2 operations per weight byte, and what counts is bytes under way.  The tensor-core
// kernel needs a tile of 64 or 128 weight rows per CTA, too few tiles for every SM when four experts are touched.
#include "linear.cuh"

namespace mcce {
namespace linear {
namespace {

constexpr int kStep = 256;    // reduction per step of a warp: 8 bf16 per lane
constexpr int kAhead = 4;     // steps under way.  With one row and 3 CTAs per SM, us for 4 x 2 x 1408 x 2048 / 1 x 14336 x 4096: 12.7 / 24.2; 8 steps, 2 CTAs: 14.7 / 22.2;
                              // 3 steps, 4 CTAs: 14.9 / 25.1

// Weights: no reuse, past L1.  Not through the read-only path: an optimiser's kernel may still be writing them when this one takes its place.
__device__ __forceinline__ uint4 read_once(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void dot_8(const uint4& a, const uint4& b, float& s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
    s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
  }
}

// M rows of x times this warp's weight rows: one feature of a gated layer (two weight rows), or two features.
template <bool GATED, int M>
__device__ __forceinline__ void few_rows(const Problem& p, int g, int64_t row, int f) {
  const int lane = threadIdx.x & 31;
  const __nv_bfloat16* w0 = (const __nv_bfloat16*)p.w + g * p.step_w + (int64_t)f * p.ld_w;
  const bool second = GATED || f + 1 < p.n;
  const __nv_bfloat16* w1 = GATED ? (const __nv_bfloat16*)p.w_up + g * p.step_w + (int64_t)f * p.ld_w : second ? w0 + p.ld_w : w0;
  const __nv_bfloat16* x = (const __nv_bfloat16*)p.x + row * p.ld_x;
  float s[2][M] = {};
  for (int k0 = 8 * lane; k0 < p.k; k0 += kStep * kAhead) {
    uint4 a[kAhead], b[kAhead], v[kAhead][M];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = k0 + kStep * i;
      const bool in = k < p.k;   // k is a multiple of 8, and so is p.k
      a[i] = in ? read_once(w0 + k) : make_uint4(0u, 0u, 0u, 0u);
      b[i] = in ? read_once(w1 + k) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int m = 0; m < M; ++m) v[i][m] = in ? *(const uint4*)(x + m * p.ld_x + k) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int m = 0; m < M; ++m) dot_8(a[i], v[i][m], s[0][m]), dot_8(b[i], v[i][m], s[1][m]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int d = 16; d; d /= 2) s[i][m] += __shfl_xor_sync(0xffffffffu, s[i][m], d);
  // lane 2 m + i has row m, and of an ungated layer feature f + i
  float z = 0.f, up = 0.f;
#pragma unroll
  for (int m = 0; m < M; ++m)
    if (lane >> 1 == m) z = GATED || (lane & 1) == 0 ? s[0][m] : s[1][m], up = s[1][m];
  if (lane >= 2 * M || (GATED ? (lane & 1) != 0 : (lane & 1) != 0 && !second)) return;
  const ForwardArgs& e = p.fwd;
  typedef __nv_bfloat16 T;
  f += GATED ? 0 : lane & 1, row += lane >> 1;
  if (e.bias) {
    const int64_t at = (int64_t)g * p.n + f;
    z += e.bias_f32 ? ((const float*)e.bias)[at] : load_as_float((const T*)e.bias + at);
    if (GATED) up += e.bias_f32 ? ((const float*)e.bias_up)[at] : load_as_float((const T*)e.bias_up + at);
  }
  if (e.saved) {
    store_as((T*)e.saved + row * e.ld_saved + f, z);
    if (GATED) store_as((T*)e.saved + row * e.ld_saved + p.n + f, up);
  }
  float y = z;
  if (e.act == MCCE_ACT_SILU) y *= e.out_f32 ? sigmoid_wide(z) : sigmoid<true>(z);
  else if (e.act == MCCE_ACT_GELU) y *= normcdff(z);
  if (GATED) y *= up;
  if (e.out_f32) {
    if (e.add) y += ((const float*)e.add)[row * e.ld_add + f];
    ((float*)e.out)[row * e.ld_out + f] = y;
  } else {
    if (e.add) y += load_as_float((const T*)e.add + row * e.ld_add + f);
    store_as((T*)e.out + row * e.ld_out + f, y);
  }
}

// M rows of x at a time; more rows of an expert read its weights again (from L2).
template <bool GATED, int M>
__global__ void __launch_bounds__(256, M == 1 ? 3 : 2) few_kernel(const __grid_constant__ Problem p) {
  extern __shared__ int before[];
  after_previous();
  count_tiles(p.groups, M, before, before + p.groups.G + 1);
  const int FT = GATED ? p.n : (p.n + 1) / 2;
  const int64_t items = (int64_t)before[p.groups.G] * FT;
  for (int64_t w = blockIdx.x * 8ll + (threadIdx.x >> 5); w < items; w += gridDim.x * 8ll) {
    const int tile = (int)(w / FT), f = (int)(w % FT) * (GATED ? 1 : 2);
    const int g = find_group(before, p.groups.G, tile);
    const GroupRows gr = group_rows(p.groups, g);
    const int in = (tile - before[g]) * M, m = (int)min((int64_t)M, gr.m - in);
    const int64_t row = gr.first + in;
    if (M == 1 || m == 1) few_rows<GATED, 1>(p, g, row, f);
    else if (m == 2) few_rows<GATED, 2>(p, g, row, f);
    else if (m == 3) few_rows<GATED, 3>(p, g, row, f);
    else few_rows<GATED, 4>(p, g, row, f);
  }
}

template <bool GATED, int M>
cudaError_t launch_few(const Problem& p, int sms, cudaStream_t st) {
  const int64_t rows = p.L * p.groups.R, tiles = rows < p.groups.G ? rows : rows / M + p.groups.G;
  const int64_t want = (tiles * (GATED ? p.n : (p.n + 1) / 2) + 7) / 8, most = (M == 1 ? 3 : 2) * sms;
  return launch_close(few_kernel<GATED, M>, dim3((unsigned)(want < most ? want : most)), 256, (size_t)(p.groups.G + 1 + 33) * 4, st, 1, p);
}

}  // namespace

// Up to four rows per expert on average, and too few tiles for the tensor-core kernel to occupy the SMs, alone or sharing a reduction.  us here / there, rows x k x n of
// one expert, and gated layers 2048 -> 1408 (222 tiles: 10 touched experts):
//   1 x 2048 x 4096: 6 / 10      1 x 14336 x 4096: 22 / 27     1 x 4096 x 16384: 24 / 27      1 token x 4 experts: 10.9 / 14.5
//   4 x 2048 x 4096: 7 / 10      4 x 14336 x 4096: 30 / 27     4 x 4096 x 16384: 36 / 27      2 tokens: 17.0 / 25.5
//   2 x 14336 x 4096: 23 / 27    3 x 14336 x 4096: 26 / 27     2 x 4096 x 16384: 28 / 27      4 tokens (too many tiles): 31.3 / 30.6
// So three or four rows of one wide expert would be better off there (up to 9 us); the rule does not look at rows and width together.
bool few_applicable(const Problem& p, int32_t dtype) {
  const uintptr_t all = (uintptr_t)p.x | (uintptr_t)p.w | (uintptr_t)p.w_up | (uintptr_t)(p.ld_x * 2) | (uintptr_t)(p.ld_w * 2) |
                        (uintptr_t)(p.groups.G > 1 ? p.step_w * 2 : 0);
  const int64_t rows = p.L * p.groups.R, G = p.groups.G, tiles = (rows < G ? rows : G) * ((p.n + (p.gated ? 63 : 127)) / (p.gated ? 64 : 128));
  return dtype == MCCE_BF16 && (all & 15) == 0 && p.k % 8 == 0 && !p.fwd.scales && rows <= 4 * G && tiles < 222;
}
cudaError_t run_few(const Problem& p, cudaStream_t st) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaErrorInvalidDevice;
  if (p.L * p.groups.R <= p.groups.G / 4 || p.L * p.groups.R == 1)
    return p.gated ? launch_few<true, 1>(p, sms, st) : launch_few<false, 1>(p, sms, st);
  return p.gated ? launch_few<true, 4>(p, sms, st) : launch_few<false, 4>(p, sms, st);
}

}  // namespace linear
}  // namespace mcce
