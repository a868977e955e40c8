// Root-mean-square norm of the residual stream with the residual's addition and, optionally, 8-bit rows with
// scales; and its gradient.
#include <cuda_fp8.h>
#include <math.h>

#include "common.cuh"
#include "vec.cuh"

namespace mcce {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMaxNormD = 16384;
constexpr int kThreads = 256;
constexpr float kE4m3Max = 448.f;
constexpr uint32_t kAmaxFloor = 0x0d800000u;   // bits of 2^-100

struct NormArgs {
  int64_t rows, ld_x, ld_add, ld_sum, ld_out, ld_q;
  int d, group, n_groups, add_f32, weight_f32;
  float eps;
  const void *x, *add, *weight;
  void *sum, *out;
  uint8_t* q;
  float* scales;
};

__device__ __forceinline__ float block_sum(float v, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < kThreads / 32; ++i) s += buf[i];
  return s;
}

template <typename T>
__device__ __forceinline__ float get1(const void* p, int64_t i, int f32) {
  if (f32 || sizeof(T) == 4) return ((const float*)p)[i];
  return __bfloat162float(((const __nv_bfloat16*)p)[i]);
}
template <typename T>
__device__ __forceinline__ T round1(float v) {
  if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v);
  else return v;
}
template <typename T>
__device__ __forceinline__ float wide1(T v) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(v);
  else return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_kernel(const NormArgs a) {
  __shared__ float buf[kThreads / 32];
  __shared__ uint32_t amax[kMaxNormD / 32];
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.x + r * a.ld_x;
  T* sum = a.sum ? (T*)a.sum + r * a.ld_sum : nullptr;
  for (int g = threadIdx.x; g < a.n_groups; g += kThreads) amax[g] = kAmaxFloor;
  float ss = 0.f;
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    float h = wide1(x[j]);
    if (a.add) h = wide1(round1<T>(h + get1<T>(a.add, r * a.ld_add + j, a.add_f32)));
    if (sum) sum[j] = round1<T>(h);
    ss = fmaf(h, h, ss);
  }
  const float inv = 1.f / sqrtf(block_sum(ss, buf) / (float)a.d + a.eps);
  auto n_at = [&](int j) {
    float h = sum ? wide1(sum[j]) : wide1(x[j]);
    if (!sum && a.add) h = wide1(round1<T>(h + get1<T>(a.add, r * a.ld_add + j, a.add_f32)));
    return h * inv * get1<T>(a.weight, j, a.weight_f32);
  };
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    const float n = n_at(j);
    if (a.out) ((T*)a.out)[r * a.ld_out + j] = round1<T>(n);
    if (a.q) atomicMax(&amax[j / a.group], __float_as_uint(fabsf(n)));
  }
  if (!a.q) return;
  __syncthreads();
  for (int g = threadIdx.x; g < a.n_groups; g += kThreads)
    a.scales[r * a.n_groups + g] = __uint_as_float(amax[g]) / kE4m3Max;
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    const float s = __uint_as_float(amax[j / a.group]) / kE4m3Max;
    a.q[r * a.ld_q + j] = __nv_cvt_float_to_fp8(n_at(j) / s, __NV_SATFINITE, __NV_E4M3);
  }
}

struct NormGradArgs {
  int64_t rows, ld_dout, ld_h, ld_dsum, ld_dx;
  int d, weight_f32, parts;
  float eps;
  const void *dout, *h, *dsum, *weight;
  void* dx;
  float* part;   // [parts, d]
};

template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_grad_kernel(const NormGradArgs a) {
  __shared__ float buf[kThreads / 32];
  float* part = a.part ? a.part + (int64_t)blockIdx.x * a.d : nullptr;
  if (part)
    for (int j = threadIdx.x; j < a.d; j += kThreads) part[j] = 0.f;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *g = (const T*)a.dout + r * a.ld_dout, *h = (const T*)a.h + r * a.ld_h;
    float ss = 0.f, sg = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float hj = wide1(h[j]);
      ss = fmaf(hj, hj, ss);
      sg = fmaf(hj, wide1(g[j]) * get1<T>(a.weight, j, a.weight_f32), sg);
    }
    const float inv = 1.f / sqrtf(block_sum(ss, buf) / (float)a.d + a.eps);
    const float coef = inv * inv * inv * (block_sum(sg, buf) / (float)a.d);
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
      const float hj = wide1(h[j]), gj = wide1(g[j]);
      float v = inv * (gj * get1<T>(a.weight, j, a.weight_f32)) - hj * coef;
      if (a.dsum) v += wide1(((const T*)a.dsum)[r * a.ld_dsum + j]);
      ((T*)a.dx)[r * a.ld_dx + j] = round1<T>(v);
      if (part) part[j] += gj * (hj * inv);
    }
  }
}

__global__ void dweight_kernel(const float* part, float* dweight, int parts, int d) {
  const int j = blockIdx.x * blockDim.x + threadIdx.x;
  if (j >= d) return;
  float s = 0.f;
  for (int p = 0; p < parts; ++p) s += part[(int64_t)p * d + j];
  dweight[j] = s;
}

constexpr int kMaxParts = 592;
int grad_parts(const mcce_norm& n) { return n.rows < kMaxParts ? (int)n.rows : kMaxParts; }

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
int64_t ld_or(int64_t ld, int d) { return ld ? ld : d; }

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
  const size_t e = elem(n->dtype);
  if (!aligned(x, e) || !aligned(sum, e) || !aligned(out, e) || !aligned(weight, elem(n->weight_dtype)) ||
      (add && !aligned(add, elem(n->add_dtype))) || !aligned(scales, 4))
    return MCCE_EINVAL;
  if (sum == x && ld_or(n->ld_sum, n->d) != ld_or(n->ld_x, n->d)) return MCCE_EINVAL;
  NormArgs a;
  a.rows = n->rows, a.d = n->d, a.eps = n->eps;
  a.ld_x = ld_or(n->ld_x, n->d), a.ld_add = ld_or(n->ld_add, n->d), a.ld_sum = ld_or(n->ld_sum, n->d);
  a.ld_out = ld_or(n->ld_out, n->d), a.ld_q = ld_or(n->ld_q, n->d);
  a.group = q ? (g ? g : n->d) : n->d, a.n_groups = q ? (n->d + a.group - 1) / a.group : 0;
  a.add_f32 = n->add_dtype == MCCE_F32, a.weight_f32 = n->weight_dtype == MCCE_F32;
  a.x = x, a.add = add, a.weight = weight, a.sum = sum, a.out = out, a.q = (uint8_t*)q, a.scales = scales;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (n->dtype == MCCE_F32) rmsnorm_kernel<float><<<(unsigned)n->rows, kThreads, 0, st>>>(a);
  else rmsnorm_kernel<__nv_bfloat16><<<(unsigned)n->rows, kThreads, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}

extern "C" size_t mcce_rmsnorm_backward_workspace_bytes(const mcce_norm* n) {
  return norm_ok(n) ? (size_t)(n->rows ? grad_parts(*n) : 1) * n->d * 4 : 0;
}

extern "C" int mcce_rmsnorm_backward(const mcce_norm* n, const void* dout, const void* h, const void* dsum,
                                     const void* weight, void* dx, float* dweight, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream) {
  if (!norm_ok(n) || (n->rows && (!dout || !h || !weight || !dx))) return MCCE_EINVAL;
  const size_t e = elem(n->dtype);
  if (!aligned(dout, e) || !aligned(h, e) || !aligned(dsum, e) || !aligned(dx, e) ||
      !aligned(weight, elem(n->weight_dtype)) || !aligned(dweight, 4))
    return MCCE_EINVAL;
  NormGradArgs a;
  a.rows = n->rows, a.d = n->d, a.eps = n->eps, a.weight_f32 = n->weight_dtype == MCCE_F32;
  a.ld_dout = ld_or(n->ld_out, n->d), a.ld_h = ld_or(n->ld_x, n->d), a.ld_dsum = ld_or(n->ld_add, n->d);
  a.ld_dx = ld_or(n->ld_sum, n->d);
  if ((dx == dout && a.ld_dx != a.ld_dout) || (dx == dsum && a.ld_dx != a.ld_dsum)) return MCCE_EINVAL;
  if (dweight) {
    if (!workspace || !aligned(workspace, 16)) return MCCE_EINVAL;
    if (workspace_bytes < mcce_rmsnorm_backward_workspace_bytes(n)) return MCCE_ENOSPC;
  }
  cudaStream_t st = (cudaStream_t)cuda_stream;
  a.dout = dout, a.h = h, a.dsum = dsum, a.weight = weight, a.dx = dx, a.part = dweight ? (float*)workspace : nullptr;
  a.parts = grad_parts(*n);
  if (a.parts) {
    if (n->dtype == MCCE_F32) rmsnorm_grad_kernel<float><<<a.parts, kThreads, 0, st>>>(a);
    else rmsnorm_grad_kernel<__nv_bfloat16><<<a.parts, kThreads, 0, st>>>(a);
  }
  if (dweight) dweight_kernel<<<(n->d + 127) / 128, 128, 0, st>>>(a.part, dweight, a.parts, n->d);
  return cudaGetLastError() == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
