// Root-mean-square norm of the residual stream with the residual's addition and, optionally, 8-bit rows with
// scales; and its gradient.
#include <cuda_fp8.h>
#include <math.h>

#include "common.cuh"
#include "tc_common.cuh"
#include "vec.cuh"

namespace mcce {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMaxNormD = MCCE_NORM_MAX_D;
constexpr float kE4m3Max = 448.f;
constexpr uint32_t kAmaxFloor = 0x0d800000u;   // bits of 2^-100

// ---- threads of a row: a power of two up to a warp (several rows per CTA), or the whole CTA -------------------
struct RowThreads {
  int tpr, t, slot;   // threads per row, this thread's index in its row, row of the CTA
  __device__ __forceinline__ explicit RowThreads(int tpr_) : tpr(tpr_) {
    if (tpr > 32) t = threadIdx.x, slot = 0;
    else t = threadIdx.x & (tpr - 1), slot = threadIdx.x / (unsigned)tpr;
  }
};

template <typename V, typename F>
__device__ __forceinline__ V row_reduce(V v, int tpr, V* buf, V neutral, F op) {
  if (tpr < 32) {
    for (int o = tpr >> 1; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kFull, v, o));
    return v;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kFull, v, o));
  if (tpr == 32) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? buf[lane] : neutral;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
// buf: one word per warp, not used again before the next barrier
__device__ __forceinline__ float row_sum(float v, int tpr, float* buf) {
  return row_reduce(v, tpr, buf, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ uint32_t row_max(uint32_t v, int tpr, uint32_t* buf) {
  return row_reduce(v, tpr, buf, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// ---- forward ------------------------------------------------------------------------------------------------------
enum Quant { kQuantRow = 1, kQuantLanes = 2, kQuantShared = 3 };   // how the largest magnitude of a group is found

struct NormArgs {
  int64_t rows, ld_x, ld_add, ld_sum, ld_out, ld_q;
  int d, n_groups, group_log2, tpr, off, add_f32, weight_f32;
  int quant;
  float eps, inv_d;
  const void *x, *add, *weight;
  void *sum, *out;
  uint8_t* q;
  float* scales;
};

// r of the norm (rsqrtf is within 2 units in the last place)
__device__ __forceinline__ float inv_rms(float sum_sq, float inv_d, float eps) { return rsqrtf(fmaf(sum_sq, inv_d, eps)); }
// scale of a group from the bits of its largest magnitude, and what its values are multiplied by.  Both are one correctly rounded
// division; the factor comes from the largest magnitude itself, not from the rounded scale, so a value is off by
// two roundings before the one to 8 bits.  (With an approximate reciprocal of a scale formed with a rounded 1 / 448 it was up to 7.)
// Codes that differ from the quotient in 64 bits: 12 of 8.4 million in groups of 128 (the plain form in fp32: 9), fp32 in groups of 32
// 49 of 67 million (56).
__device__ __forceinline__ float scale_of(uint32_t amax) { return __fdiv_rn(__uint_as_float(amax), kE4m3Max); }
__device__ __forceinline__ float back_of(uint32_t amax) { return __fdiv_rn(kE4m3Max, __uint_as_float(amax)); }

__device__ __forceinline__ uint8_t e4m3(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }
template <int N>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float2 (&v)[N]) {
  __nv_fp8x2_storage_t e[N];
#pragma unroll
  for (int j = 0; j < N; ++j) e[j] = __nv_cvt_float2_to_fp8x2(v[j], __NV_SATFINITE, __NV_E4M3);
  typename RawOf<2 * N>::type raw;
  memcpy(&raw, e, sizeof(raw));
  *(typename RawOf<2 * N>::type*)p = raw;
}
__device__ __forceinline__ uint32_t magnitude(float n) { return __float_as_uint(fabsf(n)); }   // NaN above everything

// Column of the single element that thread t of a ragged row looks after: the first U threads before the units, the next U behind.
template <int U>
__device__ __forceinline__ int single_column(int t, int head, int whole, int d) {
  const int c = t < U ? t : head + whole + t - U;
  return (t < U ? t < head : t < 2 * U && c < d) ? c : -1;
}

// A row is read once: its units stay in registers from the addition to the last output, VPT of them per thread, so
// that a thread has all its loads in flight before the point where the threads of a row meet.  fp32 arithmetic in pairs: one
// element at a time, with its conversions, kept the scheduler busier than the memory (16384 x 4096 bf16: 98 us, now 81.5).
// Bound: HBM, 1.0 of the copy bandwidth there (537 MB); ragged rows 0.91 (16384 x 4097 bf16: 90 us; with fp32 add and 8-bit rows 148, 0.76)
// and rows aligned unlike each other, in the kernel below, 0.39 (16384 x 4096: 209 us).
// RAGGED: rows start anywhere.  The units are those of the memory, up to U - 1 elements before the first and behind
// the last one are single elements, one for each of the row's first 2 U threads.
template <typename T, typename A, typename W, int VPT, bool RAGGED>
__global__ void __launch_bounds__(512) rmsnorm_kernel(const __grid_constant__ NormArgs a) {
  constexpr int U = 16 / (int)sizeof(T);
  __shared__ float buf[32];
  __shared__ uint32_t buf_max[32];
  __shared__ uint32_t amax[RAGGED ? kMaxNormD / 32 : 1];
  const RowThreads th(a.tpr);
  const int64_t r = a.tpr > 32 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / a.tpr) + th.slot;
  const int d = r < a.rows ? a.d : 0;
  const int head = RAGGED ? min(d, (int)(-(r * a.ld_x + a.off) & (U - 1))) : 0;
  const int whole = RAGGED ? (d - head) & ~(U - 1) : d;   // columns in units
  const int c0 = th.t * U, step = a.tpr * U;
  bool in[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) in[i] = c0 + i * step < whole;
  if (RAGGED && a.quant == kQuantShared) {
    for (int g = threadIdx.x; g < (int)(blockDim.x / a.tpr) * a.n_groups; g += blockDim.x) amax[g] = kAmaxFloor;
    __syncthreads();
  }

  // ---- h = x + add ------------------------------------------------------------------------------------------------
  Pack<T, U> h[VPT];
  const T* xr = (const T*)a.x + r * a.ld_x;
  const A* ar = (const A*)a.add + r * a.ld_add;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    h[i].zero();
    if (in[i]) h[i].load(xr + head + c0 + i * step);
  }
  if (a.add) {
    Pack<A, U> y[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      y[i].zero();
      if (in[i]) y[i].load(ar + head + c0 + i * step);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 v[U / 2], w[U / 2];
      h[i].get(v);
      y[i].get(w);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) v[j] = add2(v[j], w[j]);
      h[i].set(v);
    }
  }
  const int ce = RAGGED ? single_column<U>(th.t, head, whole, d) : -1;   // of this thread's single element, -1: none
  float he = 0.f;
  if (ce >= 0) {
    he = wide(xr[ce]);
    if (a.add) he = wide(narrow<T>(he + wide(ar[ce])));
  }
  float2 ss2 = make_float2(he * he, 0.f);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    float2 v[U / 2];
    h[i].get(v);
#pragma unroll
    for (int j = 0; j < U / 2; ++j) ss2 = fma2(v[j], v[j], ss2);
  }
  const float ss = ss2.x + ss2.y;
  if (a.sum) {
    T* sum = (T*)a.sum + r * a.ld_sum;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (in[i]) h[i].store(sum + head + c0 + i * step);
    if (ce >= 0) sum[ce] = narrow<T>(he);
  }
  if (!a.out && !a.q) return;

  // ---- n = h r weight ---------------------------------------------------------------------------------------------
  const W* weight = (const W*)a.weight;
  Pack<W, U> w[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) w[i].zero();
  auto load_weights = [&](auto how) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (in[i]) load_shifted<W, U, decltype(how)::value>(w[i], weight + head + c0 + i * step);
  };
  if constexpr (RAGGED) with_shift(weight + head, whole, weight, weight + a.d, load_weights);
  else load_weights(Int<kInPlace>{});
  const float we = ce >= 0 ? wide(weight[ce]) : 0.f;
  const float inv = inv_rms(row_sum(ss, a.tpr, buf), a.inv_d, a.eps);
  const float ne = he * inv * we;
  auto norm_unit = [&](int i, float2 (&n)[U / 2]) {
    float2 wv[U / 2];
    h[i].get(n);
    w[i].get(wv);
#pragma unroll
    for (int j = 0; j < U / 2; ++j) n[j] = mul2(mul2(n[j], both(inv)), wv[j]);
  };
  if (a.out) {
    T* out = (T*)a.out + r * a.ld_out;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 n[U / 2];
      norm_unit(i, n);
      Pack<T, U> o;
      o.set(n);
      if (in[i]) o.store(out + head + c0 + i * step);
    }
    if (ce >= 0) out[ce] = narrow<T>(ne);
  }
  if (!a.q) return;

  // ---- 8-bit rows -------------------------------------------------------------------------------------------------
  uint8_t* q = a.q + r * a.ld_q;
  float* scales = a.scales + r * a.n_groups;
  if (a.quant == kQuantRow) {
    uint32_t top = max(kAmaxFloor, magnitude(ne));
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 n[U / 2];
      norm_unit(i, n);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) top = max(top, max(magnitude(n[j].x), magnitude(n[j].y)));
    }
    top = row_max(top, a.tpr, buf_max);
    const float back = back_of(top);
    if (d && th.t == 0) scales[0] = scale_of(top);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 n[U / 2];
      norm_unit(i, n);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) n[j] = mul2(n[j], both(back));
      if (in[i]) store_e4m3(q + head + c0 + i * step, n);
    }
    if (ce >= 0) q[ce] = e4m3(ne * back);
  } else if (!RAGGED) {
    // A group is a power of two of neighbouring lanes, at least VPT of them: lane i does the two divisions for the group that the
    // i-th units lie in.  In every lane, for every unit, 16384 x 4096 bf16 in groups of 32 takes
    // 100 us, so 93.
    const int lanes = (1 << a.group_log2) / U, me = th.t & (lanes - 1);
    uint32_t top = kAmaxFloor;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 n[U / 2];
      norm_unit(i, n);
      uint32_t m = kAmaxFloor;
#pragma unroll
      for (int j = 0; j < U / 2; ++j) m = max(m, max(magnitude(n[j].x), magnitude(n[j].y)));
      for (int o = lanes >> 1; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(kFull, m, o));
      if (me == i) top = m;
    }
    const float back = back_of(top);
    const int cg = c0 - me * U + me * step;   // first column of that group
    if (me < VPT && cg < whole) scales[cg >> a.group_log2] = scale_of(top);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float2 n[U / 2];
      norm_unit(i, n);
      const float b = __shfl_sync(kFull, back, ((int)threadIdx.x & 31 & ~(lanes - 1)) + i);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) n[j] = mul2(n[j], both(b));
      if (in[i]) store_e4m3(q + c0 + i * step, n);
    }
  } else {
    // a unit's columns may belong to two groups
    uint32_t* m = amax + th.slot * a.n_groups;
    if (ce >= 0) atomicMax(m + (ce >> a.group_log2), magnitude(ne));
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!in[i]) continue;
      float2 n[U / 2];
      norm_unit(i, n);
      const int c = head + c0 + i * step, g = c >> a.group_log2, cut = ((g + 1) << a.group_log2) - c;
      uint32_t lo = 0, hi = 0;
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const uint32_t v = magnitude(j & 1 ? n[j / 2].y : n[j / 2].x);
        if (j < cut) lo = max(lo, v);
        else hi = max(hi, v);
      }
      atomicMax(m + g, lo);
      if (cut < U) atomicMax(m + g + 1, hi);
    }
    __syncthreads();
    if (d)
      for (int g = th.t; g < a.n_groups; g += a.tpr) {
        const uint32_t top = m[g];
        scales[g] = scale_of(top);
        m[g] = __float_as_uint(back_of(top));   // only this thread looks at it before the barrier
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!in[i]) continue;
      float2 n[U / 2];
      norm_unit(i, n);
      const int c = head + c0 + i * step, g = c >> a.group_log2, cut = ((g + 1) << a.group_log2) - c;
      const float b0 = __uint_as_float(m[g]), b1 = cut < U ? __uint_as_float(m[g + 1]) : b0;
#pragma unroll
      for (int j = 0; j < U / 2; ++j) n[j] = mul2(n[j], make_float2(2 * j < cut ? b0 : b1, 2 * j + 1 < cut ? b0 : b1));
      store_e4m3(q + c, n);
    }
    if (ce >= 0) q[ce] = e4m3(ne * __uint_as_float(m[ce >> a.group_log2]));
  }
}

// Tensors whose rows are not aligned alike (views with odd offsets or strides): element by element, three passes over a
// row, which comes back from L1 in the second and third.
constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float get1(const void* p, int64_t i, int f32) {
  if (f32 || sizeof(T) == 4) return ((const float*)p)[i];
  return __bfloat162float(((const __nv_bfloat16*)p)[i]);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_scalar_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float buf[32];
  __shared__ uint32_t amax[kMaxNormD / 32];
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.x + r * a.ld_x;
  T* sum = a.sum ? (T*)a.sum + r * a.ld_sum : nullptr;
  for (int g = threadIdx.x; g < a.n_groups; g += kThreads) amax[g] = kAmaxFloor;
  float ss = 0.f;
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    float h = wide(x[j]);
    if (a.add) h = wide(narrow<T>(h + get1<T>(a.add, r * a.ld_add + j, a.add_f32)));
    if (sum) sum[j] = narrow<T>(h);
    ss = fmaf(h, h, ss);
  }
  const float inv = inv_rms(row_sum(ss, kThreads, buf), a.inv_d, a.eps);
  auto n_at = [&](int j) {
    float h = sum ? wide(sum[j]) : wide(x[j]);
    if (!sum && a.add) h = wide(narrow<T>(h + get1<T>(a.add, r * a.ld_add + j, a.add_f32)));
    return h * inv * get1<T>(a.weight, j, a.weight_f32);
  };
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    const float n = n_at(j);
    if (a.out) ((T*)a.out)[r * a.ld_out + j] = narrow<T>(n);
    if (a.q) atomicMax(&amax[j >> a.group_log2], magnitude(n));
  }
  if (!a.q) return;
  __syncthreads();
  for (int g = threadIdx.x; g < a.n_groups; g += kThreads) {
    const uint32_t top = amax[g];
    a.scales[r * a.n_groups + g] = scale_of(top);
    amax[g] = __float_as_uint(back_of(top));
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.d; j += kThreads)
    a.q[r * a.ld_q + j] = e4m3(n_at(j) * __uint_as_float(amax[j >> a.group_log2]));
}

// How a row is laid over threads: `vpt` units for each of tpr threads.
struct NormShape {
  int tpr, vpt, threads;
};

int pow2_up(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

NormShape shape_for(int units, int vpt, int least) {
  const int need = (units + vpt - 1) / vpt > least ? (units + vpt - 1) / vpt : least;
  NormShape s;
  s.vpt = vpt;
  s.tpr = need > 32 ? (need + 31) / 32 * 32 : pow2_up(need);
  s.threads = s.tpr > 32 ? s.tpr : 128;
  return s;
}

template <typename T, typename A, typename W, int VPT>
cudaError_t launch_norm(NormArgs a, bool ragged, const NormShape& sh, cudaStream_t st) {
  a.tpr = sh.tpr;
  a.quant = !a.q ? 0 : a.n_groups == 1 ? kQuantRow : ragged ? kQuantShared : kQuantLanes;
  const int rpb = sh.threads / a.tpr;
  const unsigned grid = (unsigned)((a.rows + rpb - 1) / rpb);
  if (ragged) rmsnorm_kernel<T, A, W, VPT, true><<<grid, sh.threads, 0, st>>>(a);
  else rmsnorm_kernel<T, A, W, VPT, false><<<grid, sh.threads, 0, st>>>(a);
  return cudaGetLastError();
}
template <typename T, typename A, typename W>
cudaError_t launch_norm_vpt(const NormArgs& a, bool ragged, const NormShape& sh, cudaStream_t st) {
  constexpr int kWide = sizeof(T) == 4 ? 8 : 4;
  if (sh.vpt == 2) return launch_norm<T, A, W, 2>(a, ragged, sh, st);
  return launch_norm<T, A, W, kWide>(a, ragged, sh, st);
}
cudaError_t launch_norm_types(const NormArgs& a, int dtype, bool ragged, const NormShape& sh, cudaStream_t st) {
  using B = __nv_bfloat16;
  if (dtype == MCCE_F32) return launch_norm_vpt<float, float, float>(a, ragged, sh, st);
  if (a.add && a.add_f32) return a.weight_f32 ? launch_norm_vpt<B, float, float>(a, ragged, sh, st)
                                              : launch_norm_vpt<B, float, B>(a, ragged, sh, st);
  return a.weight_f32 ? launch_norm_vpt<B, B, float>(a, ragged, sh, st) : launch_norm_vpt<B, B, B>(a, ragged, sh, st);
}

// Two units per thread; 64 bytes of every tensor per thread (4 units of bf16, 8 of fp32) where two would need more than 512
// threads for a row, and for many wide ragged rows, whose single elements and shifted weights cost a thread the same for two units
// as for four.  us with the residual's addition (calls back to back on three sets of inputs in turn, as all figures of this file), two
// / wide: 16384 x 4096 bf16 81.5 / 82.1 (1.00 of the copy bandwidth), 16384 x 2048 with 8-bit rows 58.9 / 59.6, 131072 x 64 14.0 /
// 15.2, with 8-bit rows 20.6 / 30.8; ragged 16384 x 4098 bf16 92.9 / 90.2, 16384 x 4097 fp32 178 / 160, 4097 bf16 with fp32 add and only
// 8-bit rows 125 / 118, with out and fp32 weights beside them 143 / 148 (106 registers: the one that loses).  One unit per thread: 16384
// x 4096 84.0, 16384 x 2048 with 8-bit rows 63.6, ragged 16384 x 4098 137.
NormShape norm_shape(int64_t rows, int d, bool ragged, int elem_bytes, int group_log2) {
  const int u = 16 / elem_bytes, units = d / u;
  // a group of columns has to fit the lanes of one unit step; a ragged row needs 2 U threads for its single elements
  const int least = ragged ? 2 * u : group_log2 < 30 ? (1 << group_log2) / u : 1;
  const bool two = units <= 1024 && !(ragged && rows > 4096 && units > 256);
  return shape_for(units, two ? 2 : elem_bytes == 4 ? 8 : 4, least);
}

// ---- gradient -----------------------------------------------------------------------------------------------------
struct NormGradArgs {
  int64_t rows, ld_dout, ld_h, ld_dsum, ld_dx;
  int d, weight_f32, tpr, off, stages;
  float eps, inv_d;
  const void *dout, *h, *dsum, *weight;
  void* dx;
  float* part;   // [CTAs, d], or null: the weight's gradient is not wanted
};

// dx = r g + (h r) c + dsum with c = -r^2 mean(h g), for the vector and the scalar kernel alike.  The mean takes in one r at a time: it is
// at most as large as rms(h) rms(g), so every product on the way lies between the mean, rms(g) and c, in fp32's range where r^2 or
// r^3 alone are not.
__device__ __forceinline__ float grad_coef(float inv, float mean_hg) { return -inv * (inv * mean_hg); }

// Both sums at once: the lower half of a group of lanes ends up with x, the upper half with y.
__device__ __forceinline__ float half_sum2(float2 v, int lanes) {
  const bool upper = threadIdx.x & (lanes >> 1);
  const float got = __shfl_xor_sync(kFull, upper ? v.x : v.y, lanes >> 1);
  float s = (upper ? v.y : v.x) + got;
  for (int o = lanes >> 2; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  return s;
}
__device__ __forceinline__ float2 row_sum2(float2 v, int tpr, float* buf) {   // buf: two words per warp
  const int lane = threadIdx.x & 31;
  if (tpr == 1) return v;
  if (tpr < 32) {
    const float s = half_sum2(v, tpr), other = __shfl_xor_sync(kFull, s, tpr >> 1);
    return lane & (tpr >> 1) ? make_float2(other, s) : make_float2(s, other);
  }
  float s = half_sum2(v, 32);
  if (tpr > 32) {   // sixteen warps at most: x of warp w in buf[w], y in buf[16 + w]
    if ((lane & 15) == 0) buf[(lane & 16) + (threadIdx.x >> 5)] = s;
    __syncthreads();
    s = (lane & 15) < (int)(blockDim.x >> 5) ? buf[lane] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  }
  return make_float2(__shfl_sync(kFull, s, 0), __shfl_sync(kFull, s, 16));
}

// 16 bytes from global to shared memory without passing through registers.  A thread reads only what it copied itself,
// so waiting for its own copies is all the order that is needed.
__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A CTA takes rows blockIdx.x, + gridDim.x, ... (times the rows it holds at once).  The rows come through a ring of
// `stages` slots in shared memory, filled stages - 1 rows ahead: a row's two passes (the sums, then dx) hang on one
// another through a reduction over its threads, and only copies that are under way meanwhile keep the memory busy.
// RAGGED: the step between a thread's rows is a multiple of U (or it has one row), so that every one of its rows starts at
// the same place in a unit.  A thread therefore has the same columns in all its rows, aligned or not, and keeps their
// weights and its part of the weights' gradient in registers.
// Bound: HBM for aligned rows (16384 x 2048 bf16 with dsum: 43.0 us = 0.95 of the copy bandwidth, 47.6 with the launch that
// adds the parts of the weight's gradient); ragged rows add the pass over the single elements to every row's chain (16384 x 4097: 96
// us = 0.85).  With the row in registers instead of the ring, loaded when it was needed, the first took 62 us; with columns that
// move from row to row and sums in shared memory the second 148.  62 to 102 registers with two units per thread; the wide forms hold
// 128 and the aligned ones of them spill (20 bytes for bf16 above 8192 columns, 56 for fp32 above 4096: 16384 x 8192 bf16 164 us = 1.00,
// 16384 x 5120 fp32 224 us = 0.91).
template <typename T, typename W, int VPT, bool RAGGED>
__global__ void __launch_bounds__(512) rmsnorm_grad_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr int U = 16 / (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];   // the ring; at the end [rows per CTA][d] sums
  __shared__ float buf[2][32];
  const RowThreads th(a.tpr);
  const int rpb = blockDim.x / a.tpr;
  const int64_t stride = (int64_t)gridDim.x * rpb, first = (int64_t)blockIdx.x * rpb + th.slot;
  const int head = RAGGED ? min(a.d, (int)(-(first * a.ld_h + a.off) & (U - 1))) : 0;
  const int whole = RAGGED ? (a.d - head) & ~(U - 1) : a.d;
  const int c0 = th.t * U, step = a.tpr * U;
  bool in[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) in[i] = c0 + i * step < whole;
  const int tensor_bytes = VPT * (int)blockDim.x * 16, stage_bytes = (a.dsum ? 3 : 2) * tensor_bytes;
  uint8_t* ring = smem + threadIdx.x * 16;

  const int ce = RAGGED ? single_column<U>(th.t, head, whole, a.d) : -1;   // of this thread's single element, -1: none
  struct Single {
    T h, g, s;   // as loaded: converting would wait for them
  } one{}, next{};
  auto fetch_one = [&](int64_t r) {
    if (ce < 0 || r >= a.rows) return;
    next.h = ((const T*)a.h)[r * a.ld_h + ce];
    next.g = ((const T*)a.dout)[r * a.ld_dout + ce];
    if (a.dsum) next.s = ((const T*)a.dsum)[r * a.ld_dsum + ce];
  };
  auto fetch = [&](int64_t r, int stage) {
    const T *hr = (const T*)a.h + r * a.ld_h + head, *gr = (const T*)a.dout + r * a.ld_dout + head;
    const T* sr = (const T*)a.dsum + r * a.ld_dsum + head;
    uint8_t* to = ring + stage * stage_bytes;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!(r < a.rows && in[i])) {   // adds nothing to the sums
        *(uint4*)(to + i * (int)blockDim.x * 16) = *(uint4*)(to + tensor_bytes + i * (int)blockDim.x * 16) = make_uint4(0, 0, 0, 0);
        continue;
      }
      const int c = c0 + i * step;
      copy16(to + i * (int)blockDim.x * 16, hr + c);
      copy16(to + tensor_bytes + i * (int)blockDim.x * 16, gr + c);
      if (a.dsum) copy16(to + 2 * tensor_bytes + i * (int)blockDim.x * 16, sr + c);
    }
  };

  for (int k = 0; k < a.stages - 1; ++k) {
    fetch(first + k * stride, k);
    copies_commit();
  }
  if (RAGGED) fetch_one(first);
  const W* weight = (const W*)a.weight;
  float2 w[VPT][U / 2], dw[VPT][U / 2];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    Pack<W, U> p;
    p.zero();
    if (in[i]) {
      if constexpr (RAGGED) p.load_part(weight + head + c0 + i * step, 0, U);   // once per CTA
      else p.load_const(weight + c0 + i * step);
    }
    p.get(w[i]);
#pragma unroll
    for (int j = 0; j < U / 2; ++j) dw[i][j] = both(0.f);
  }
  const float we = ce >= 0 ? wide(weight[ce]) : 0.f;
  float dwe = 0.f;
  int stage = 0, par = 0;
  for (int64_t base = (int64_t)blockIdx.x * rpb; base < a.rows; base += stride, par ^= 1) {
    const int64_t r = base + th.slot;
    int into = stage + a.stages - 1;
    if (into >= a.stages) into -= a.stages;
    fetch(r + (a.stages - 1) * stride, into);
    copies_commit();
    float2 sum = both(0.f);   // of h^2, of h g
    if (RAGGED) {
      one = next;
      fetch_one(r + stride);
      const float he = wide(one.h);   // zero for a thread without one
      sum = make_float2(he * he, he * (wide(one.g) * we));
    }
    if (a.stages == 1) copies_wait<0>();
    else if (a.stages == 2) copies_wait<1>();
    else copies_wait<2>();
    const uint8_t* row = ring + stage * stage_bytes;
    float2 hh = both(0.f), hg = both(0.f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      Pack<T, U> h, g;
      h.load((const T*)(row + i * (int)blockDim.x * 16)), g.load((const T*)(row + tensor_bytes + i * (int)blockDim.x * 16));
      float2 hv[U / 2], gv[U / 2];
      h.get(hv), g.get(gv);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) {
        hh = fma2(hv[j], hv[j], hh);
        hg = fma2(hv[j], mul2(gv[j], w[i][j]), hg);
      }
    }
    sum.x += hh.x + hh.y, sum.y += hg.x + hg.y;
    sum = row_sum2(sum, a.tpr, buf[par]);
    const float inv = r < a.rows ? inv_rms(sum.x, a.inv_d, a.eps) : 0.f, coef = grad_coef(inv, sum.y * a.inv_d);
    T* xr = (T*)a.dx + r * a.ld_dx + head;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      Pack<T, U> h, g, o;
      h.load((const T*)(row + i * (int)blockDim.x * 16)), g.load((const T*)(row + tensor_bytes + i * (int)blockDim.x * 16));
      o.zero();
      if (a.dsum) o.load((const T*)(row + 2 * tensor_bytes + i * (int)blockDim.x * 16));
      float2 hv[U / 2], gv[U / 2], v[U / 2];
      h.get(hv), g.get(gv), o.get(v);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) {
        const float2 n = mul2(hv[j], both(inv));
        dw[i][j] = fma2(gv[j], n, dw[i][j]);
        v[j] = fma2(mul2(gv[j], w[i][j]), both(inv), fma2(n, both(coef), v[j]));
      }
      o.set(v);
      if (in[i] && r < a.rows) o.store(xr + c0 + i * step);
    }
    if (ce >= 0 && r < a.rows) {
      const float he = wide(one.h), ge = wide(one.g);
      xr[ce - head] = narrow<T>(fmaf(ge * we, inv, fmaf(he * inv, coef, a.dsum ? wide(one.s) : 0.f)));
      dwe = fmaf(ge, he * inv, dwe);
    }
    if (++stage == a.stages) stage = 0;
  }
  copies_wait<0>();
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * a.d;
  if (!RAGGED && rpb == 1) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (in[i])
#pragma unroll
        for (int j = 0; j < U / 2; j += 2)
          *(float4*)(part + c0 + i * step + 2 * j) = make_float4(dw[i][j].x, dw[i][j].y, dw[i][j + 1].x, dw[i][j + 1].y);
    return;
  }
  // several rows at once, or units across the columns' alignment: together through shared memory
  __syncthreads();
  float* mine = (float*)smem + (size_t)th.slot * a.d;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (in[i])
#pragma unroll
      for (int j = 0; j < U / 2; ++j) {
        float* p = mine + head + c0 + i * step + 2 * j;
        p[0] = dw[i][j].x, p[1] = dw[i][j].y;
      }
  if (ce >= 0) mine[ce] = dwe;
  __syncthreads();
  for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
    float v = 0.f;
    for (int k = 0; k < rpb; ++k) v += ((const float*)smem)[(size_t)k * a.d + c];
    part[c] = v;
  }
}

// Tensors whose rows are not aligned alike: element by element, twice over a row.  16384 x 2048 bf16 with dsum 207 us (0.20 of the
// copy bandwidth): one element per thread and load, and one row of a CTA after the other.
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_grad_scalar_kernel(const __grid_constant__ NormGradArgs a) {
  __shared__ float buf[2][32];
  float* part = a.part ? a.part + (int64_t)blockIdx.x * a.d : nullptr;
  if (part)
    for (int j = threadIdx.x; j < a.d; j += kThreads) part[j] = 0.f;
  int par = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, par ^= 1) {
    const T *g = (const T*)a.dout + r * a.ld_dout, *h = (const T*)a.h + r * a.ld_h;
    float2 s = make_float2(0.f, 0.f);
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float hj = wide(h[j]);
      s.x = fmaf(hj, hj, s.x);
      s.y = fmaf(hj, wide(g[j]) * get1<T>(a.weight, j, a.weight_f32), s.y);
    }
    s = row_sum2(s, kThreads, buf[par]);
    const float inv = inv_rms(s.x, a.inv_d, a.eps), coef = grad_coef(inv, s.y * a.inv_d);
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float hj = wide(h[j]), gj = wide(g[j]);
      const float past = a.dsum ? wide(((const T*)a.dsum)[r * a.ld_dsum + j]) : 0.f;
      ((T*)a.dx)[r * a.ld_dx + j] = narrow<T>(fmaf(gj * get1<T>(a.weight, j, a.weight_f32), inv, fmaf(hj * inv, coef, past)));
      if (part) part[j] = fmaf(gj, hj * inv, part[j]);
    }
  }
}

// dweight = the sum of the parts, in a fixed order: 16 columns per CTA, 64 threads per column, each taking every 64th part.
__global__ void __launch_bounds__(1024) dweight_kernel(const float* part, float* dweight, int parts, int d) {
  __shared__ float sum[64][17];
  const int col = threadIdx.x & 15, group = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  float s = 0.f;
  cudaGridDependencySynchronize();   // starts as the last CTAs of the kernel that writes the parts end, before its memory is flushed
  if (c < d) {
#pragma unroll 10
    for (int p = group; p < parts; p += 64) s += part[(int64_t)p * d + c];
  }
  sum[group][col] = s;
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (warp >= 16) return;
  s = sum[lane][warp] + sum[lane + 32][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  if (lane == 0 && blockIdx.x * 16 + warp < d) dweight[blockIdx.x * 16 + warp] = s;
}

cudaError_t launch_dweight(const float* part, float* dweight, int parts, int d, cudaStream_t st) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((d + 15) / 16), cfg.blockDim = dim3(1024), cfg.stream = st, cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, dweight_kernel, part, dweight, parts, d);
}

constexpr int kSms = 148;

struct GradShape {
  NormShape s;
  int ctas;     // also the number of parts
  int stages;
  size_t smem;
};
constexpr size_t kGradSmemMost = 226 * 1024;   // dynamic; the reduction buffers are static

// Shared memory of the gradient kernel with a ring of `stages` rows (the layout of its declaration).
size_t grad_smem(const NormShape& s, int stages, int d, bool ragged, bool dsum, bool dweight) {
  const size_t ring = (size_t)stages * (dsum ? 3 : 2) * s.vpt * s.threads * 16, rpb = s.threads / s.tpr;
  const size_t sums = dweight && (ragged || rpb > 1) ? rpb * d * 4 : 0;
  return ring > sums ? ring : sums;
}

GradShape grad_shape(int64_t rows, int d, Layout3 lay, int elem_bytes, bool dsum, bool dweight) {
  GradShape g;
  if (lay == kScalar) {
    g.s = NormShape{kThreads, 1, kThreads};
    g.ctas = (int)(rows < 4 * kSms ? rows : 4 * kSms);
    return g;
  }
  const bool ragged = lay == kRagged;
  const int u = 16 / elem_bytes, units = d / u;
  g.s = shape_for(units, units <= 1024 ? 2 : elem_bytes == 4 ? 8 : 4, ragged ? 2 * u : 1);
  const int rpb = g.s.threads / g.s.tpr;
  const int64_t all = (rows + rpb - 1) / rpb;
  // CTAs per SM / stages, us (16384 rows with dsum, weight's gradient included): 2048 bf16 4 / 2 47.6, 3 / 3 47.3, 4 / 3 49.8, 6 / 3 56;
  // 1024 bf16 6 / 3 27.0, 6 / 2 28.7, 8 / 3 29.6; 4096 bf16 2 / 2 85.5, 2 / 3 87.0.
  int per_sm = g.s.threads <= 64 ? 6 : g.s.threads >= 384 ? 1 : g.s.threads > 192 ? 2 : 512 / g.s.threads;
  // Two such CTAs that are left with one stage lose to one with two from 288 threads on: 8192 x 9216 fp32 197 us against 152, with
  // dsum 4096 x 10000 bf16 96 against 67, 10001 113 against 80, 8192 x 8200 fp32 213 against 194.
  if (g.s.threads > 256 && grad_smem(g.s, 2, d, ragged, dsum, dweight) > kGradSmemMost / 2) per_sm = 1;
  // A third stage is worth its longer start where less than 48 KB of rows per SM are under way without it, the rows are aligned and a
  // CTA has more than eight turns.  Two stages against three, us (calls in a graph), by turns of a CTA:
  //                             2             4             8             16            32
  //   1024 bf16 with dsum    7.5 / 7.7     9.5 / 9.7   14.7 / 15.0   23.6 / 22.9   40.9 / 39.6
  //   2048 bf16              9.1 / 9.3   11.6 / 12.0   17.0 / 17.6   26.7 / 26.7   45.3 / 44.7
  //   2048 fp32              6.5 / 6.8     8.7 / 8.9   14.6 / 14.8   23.6 / 22.7   41.7 / 38.9
  //   4096 fp32              6.3 / 6.5     8.8 / 9.0   14.9 / 14.9   24.3 / 23.0   43.0 / 39.1
  //   1411 bf16, ragged      9.7 / 9.9   11.6 / 11.9   16.6 / 17.2   25.3 / 25.9   41.7 / 42.4
  //   1411 fp32, ragged      7.7 / 8.1     9.5 / 9.7   15.1 / 15.4   23.7 / 24.1   40.2 / 40.5
  //   515 fp32 with dsum, r. 8.1 / 8.2     9.1 / 9.5   13.8 / 14.5   20.7 / 21.3   34.3 / 34.9
  const size_t flying = grad_smem(g.s, 1, d, false, dsum, false) * per_sm;
  g.stages = ragged || flying >= 48 * 1024 || all <= 8 * per_sm * kSms ? 2 : 3;
  while (g.stages > 1 && grad_smem(g.s, g.stages, d, ragged, dsum, dweight) > kGradSmemMost / per_sm) --g.stages;
  g.smem = grad_smem(g.s, g.stages, d, ragged, dsum, dweight);
  int ctas = per_sm * kSms;
  if (ragged) ctas = ctas / u * u;   // rows of a thread: a multiple of u apart
  g.ctas = (int)(all < ctas ? all : ctas);
  // a few rows one after the other in a single CTA take less time than the launch that adds several CTAs' parts
  if (dweight && all <= 4 && (!ragged || rpb % u == 0)) g.ctas = 1;
  return g;
}
int parts_most(const mcce_norm& n) {
  const int64_t most = 8 * kSms;
  return (int)(n.rows < 1 ? 1 : n.rows < most ? n.rows : most);
}

template <typename T, typename W, int VPT, bool RAGGED>
cudaError_t launch_grad(NormGradArgs a, const GradShape& g, cudaStream_t st) {
  static int cache[64] = {0};   // per kernel
  int sms = 0;
  const cudaError_t e = tc::sm_count_and_smem_optin(rmsnorm_grad_kernel<T, W, VPT, RAGGED>, kGradSmemMost, cache, &sms);
  if (e != cudaSuccess) return e;
  a.tpr = g.s.tpr, a.stages = g.stages;
  rmsnorm_grad_kernel<T, W, VPT, RAGGED><<<g.ctas, g.s.threads, g.smem, st>>>(a);
  return cudaGetLastError();
}
template <typename T, typename W>
cudaError_t launch_grad_vpt(const NormGradArgs& a, bool ragged, const GradShape& g, cudaStream_t st) {
  constexpr int kWide = sizeof(T) == 4 ? 8 : 4;
  if (g.s.vpt == 2) return ragged ? launch_grad<T, W, 2, true>(a, g, st) : launch_grad<T, W, 2, false>(a, g, st);
  return ragged ? launch_grad<T, W, kWide, true>(a, g, st) : launch_grad<T, W, kWide, false>(a, g, st);
}
cudaError_t launch_grad_types(const NormGradArgs& a, int dtype, bool ragged, const GradShape& g, cudaStream_t st) {
  using B = __nv_bfloat16;
  if (dtype == MCCE_F32) return launch_grad_vpt<float, float>(a, ragged, g, st);
  return a.weight_f32 ? launch_grad_vpt<B, float>(a, ragged, g, st) : launch_grad_vpt<B, B>(a, ragged, g, st);
}

bool stride_ok(int64_t ld, int d) { return ld == 0 || ld >= d; }

bool norm_ok(const mcce_norm* n) {
  if (!n) return false;
  if (n->rows < 0 || n->rows > 0x7fffffffll || n->d < 1 || n->d > kMaxNormD) return false;
  if (n->dtype != MCCE_F32 && n->dtype != MCCE_BF16) return false;
  if (n->weight_dtype != MCCE_F32 && n->weight_dtype != n->dtype) return false;
  if (!(n->eps >= 0.f) || !isfinite(n->eps)) return false;
  return stride_ok(n->ld_x, n->d) && stride_ok(n->ld_add, n->d) && stride_ok(n->ld_sum, n->d) &&
         stride_ok(n->ld_out, n->d);
}

bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
int elem(int dtype) { return dtype == MCCE_F32 ? 4 : 2; }
int64_t ld_or(int64_t ld, int64_t d) { return ld ? ld : d; }

}  // namespace
}  // namespace mcce

using namespace mcce;

extern "C" int mcce_rmsnorm(const mcce_norm* n, const void* x, const void* add, const void* weight, void* sum,
                            void* out, void* q, float* scales, void* cuda_stream) {
  if (!norm_ok(n)) return MCCE_EINVAL;
  if (n->rows == 0) return MCCE_OK;
  if (!x || !weight || (!sum && !out && !q) || (q == nullptr) != (scales == nullptr)) return MCCE_EINVAL;
  if (add && n->add_dtype != MCCE_F32 && n->add_dtype != n->dtype) return MCCE_EINVAL;
  const int g = n->quant_group;
  if (q && ((g != 0 && g != 32 && g != 64 && g != 128) || !stride_ok(n->ld_q, n->d))) return MCCE_EINVAL;
  const int e = elem(n->dtype), ea = elem(n->add_dtype), ew = elem(n->weight_dtype);
  if (!aligned(x, e) || !aligned(sum, e) || !aligned(out, e) || !aligned(weight, ew) || (add && !aligned(add, ea)) ||
      !aligned(scales, 4))
    return MCCE_EINVAL;
  const int64_t R = n->rows, d = n->d;
  const Span sx = row_span(x, R, ld_or(n->ld_x, d), d, e), sadd = row_span(add, R, ld_or(n->ld_add, d), d, ea);
  const Span sw = flat_span(weight, d * ew), ssum = row_span(sum, R, ld_or(n->ld_sum, d), d, e);
  const Span sout = row_span(out, R, ld_or(n->ld_out, d), d, e), sq = row_span(q, R, ld_or(n->ld_q, d), d, 1);
  const Span sscales = flat_span(scales, R * (g ? (d + g - 1) / g : 1), 4);
  if (!same_or_apart(ssum, sx) || !apart(ssum, {&sadd, &sw}) || !apart(sout, {&sx, &sadd, &sw, &ssum}) ||
      !apart(sq, {&sx, &sadd, &sw, &ssum, &sout}) || !apart(sscales, {&sx, &sadd, &sw, &ssum, &sout, &sq}))
    return MCCE_EINVAL;
  NormArgs a{};
  a.rows = n->rows, a.d = n->d, a.eps = n->eps;
  a.ld_x = ld_or(n->ld_x, n->d), a.ld_add = ld_or(n->ld_add, n->d), a.ld_sum = ld_or(n->ld_sum, n->d);
  a.ld_out = ld_or(n->ld_out, n->d), a.ld_q = ld_or(n->ld_q, n->d);
  a.group_log2 = g == 0 ? 30 : g == 32 ? 5 : g == 64 ? 6 : 7;
  a.n_groups = q ? (g ? (n->d + g - 1) / g : 1) : 0;
  a.add_f32 = n->add_dtype == MCCE_F32, a.weight_f32 = n->weight_dtype == MCCE_F32, a.inv_d = 1.f / (float)n->d;
  a.x = x, a.add = add, a.weight = weight, a.sum = sum, a.out = out, a.q = (uint8_t*)q, a.scales = scales;
  LayoutRule rule(n->d, 16 / e);
  rule.tensor(x, a.ld_x, e);
  rule.tensor(add, a.ld_add, ea);
  rule.tensor(sum, a.ld_sum, e);
  rule.tensor(out, a.ld_out, e);
  rule.tensor(q, a.ld_q, 1);
  const Layout3 lay = aligned(weight, 16) ? rule.layout() : kScalar;
  a.off = rule.off;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err;
  if (lay == kScalar) {
    if (n->dtype == MCCE_F32) rmsnorm_scalar_kernel<float><<<(unsigned)n->rows, kThreads, 0, st>>>(a);
    else rmsnorm_scalar_kernel<__nv_bfloat16><<<(unsigned)n->rows, kThreads, 0, st>>>(a);
    err = cudaGetLastError();
  } else {
    const bool ragged = lay == kRagged;
    err = launch_norm_types(a, n->dtype, ragged, norm_shape(n->rows, n->d, ragged, e, q ? a.group_log2 : 30), st);
  }
  return err == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}

extern "C" size_t mcce_rmsnorm_backward_workspace_bytes(const mcce_norm* n) {
  return norm_ok(n) ? (size_t)parts_most(*n) * n->d * 4 : 0;
}

extern "C" int mcce_rmsnorm_backward(const mcce_norm* n, const void* dout, const void* h, const void* dsum,
                                     const void* weight, void* dx, float* dweight, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream) {
  if (!norm_ok(n) || (n->rows && (!dout || !h || !weight || !dx))) return MCCE_EINVAL;
  const int e = elem(n->dtype);
  if (!aligned(dout, e) || !aligned(h, e) || !aligned(dsum, e) || !aligned(dx, e) ||
      !aligned(weight, elem(n->weight_dtype)) || !aligned(dweight, 4))
    return MCCE_EINVAL;
  NormGradArgs a{};
  a.rows = n->rows, a.d = n->d, a.eps = n->eps, a.weight_f32 = n->weight_dtype == MCCE_F32, a.inv_d = 1.f / (float)n->d;
  a.ld_dout = ld_or(n->ld_out, n->d), a.ld_h = ld_or(n->ld_x, n->d), a.ld_dsum = ld_or(n->ld_add, n->d);
  a.ld_dx = ld_or(n->ld_sum, n->d);
  if (dweight) {
    if (!workspace || !aligned(workspace, 16)) return MCCE_EINVAL;
    if (workspace_bytes < mcce_rmsnorm_backward_workspace_bytes(n)) return MCCE_ENOSPC;
  }
  const int64_t R = n->rows, d = n->d;
  const Span sg = row_span(dout, R, a.ld_dout, d, e), sh = row_span(h, R, a.ld_h, d, e), sds = row_span(dsum, R, a.ld_dsum, d, e);
  const Span sw = flat_span(weight, d * elem(n->weight_dtype)), sdx = row_span(dx, R, a.ld_dx, d, e), sdw = flat_span(dweight, d * 4);
  const Span sws = flat_span(dweight ? workspace : nullptr, mcce_rmsnorm_backward_workspace_bytes(n));
  if (R && (!same_or_apart(sdx, sg) || !same_or_apart(sdx, sds) || !apart(sdx, {&sh, &sw}) || !apart(sdw, {&sg, &sh, &sds, &sw, &sdx}) ||
            !apart(sws, {&sg, &sh, &sds, &sw, &sdx, &sdw})))
    return MCCE_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (n->rows == 0)
    return !dweight || cudaMemsetAsync(dweight, 0, (size_t)n->d * 4, st) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
  a.dout = dout, a.h = h, a.dsum = dsum, a.weight = weight, a.dx = dx, a.part = dweight ? (float*)workspace : nullptr;
  LayoutRule rule(n->d, 16 / e);
  rule.tensor(h, a.ld_h, e);
  rule.tensor(dout, a.ld_dout, e);
  rule.tensor(dsum, a.ld_dsum, e);
  rule.tensor(dx, a.ld_dx, e);
  const Layout3 lay = aligned(weight, 16) ? rule.layout() : kScalar;
  a.off = rule.off;
  const GradShape g = grad_shape(n->rows, n->d, lay, e, dsum != nullptr, dweight != nullptr);
  const bool direct = g.ctas == 1 && aligned(dweight, 16);   // the only part is the result
  if (direct) a.part = dweight;
  cudaError_t err;
  if (lay == kScalar) {
    if (n->dtype == MCCE_F32) rmsnorm_grad_scalar_kernel<float><<<g.ctas, kThreads, 0, st>>>(a);
    else rmsnorm_grad_scalar_kernel<__nv_bfloat16><<<g.ctas, kThreads, 0, st>>>(a);
    err = cudaGetLastError();
  } else {
    err = launch_grad_types(a, n->dtype, lay == kRagged, g, st);
  }
  if (err == cudaSuccess && dweight && !direct) err = launch_dweight(a.part, dweight, g.ctas, n->d, st);
  return err == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
