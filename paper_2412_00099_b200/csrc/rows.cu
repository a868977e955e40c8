// Token rows sorted by expert, the rows brought back to their tokens with weights (Eq. 1's sum), and its gradient.
#include "common.cuh"
#include "vec.cuh"

namespace mcce {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kSortChunk = 1024;   // pairs per CTA of the counting sort

struct SortArgs {
  int T, K, E, P, B;
  const int32_t* sel;
  int32_t *offsets, *perm, *inv, *counts;   // counts [L][B][E]
};

__global__ void __launch_bounds__(256) rows_count_kernel(const SortArgs a) {
  __shared__ int hist[kMaxE];
  const int b = blockIdx.x, l = blockIdx.y;
  for (int e = threadIdx.x; e < a.E; e += 256) hist[e] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < kSortChunk; i += 256) {
    const int64_t q = (int64_t)b * kSortChunk + i;
    if (q < a.P) {
      const int e = a.sel[(size_t)l * a.P + q];
      if ((unsigned)e < (unsigned)a.E) atomicAdd(&hist[e], 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += 256) a.counts[((size_t)l * a.B + b) * a.E + e] = hist[e];
}

__global__ void __launch_bounds__(kSortChunk) rows_rank_kernel(const SortArgs a) {
  __shared__ int total[kMaxE], before[kMaxE], warp_at[kSortChunk / 32][kMaxE];
  const int b = blockIdx.x, l = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < a.E) total[tid] = before[tid] = 0;
  for (int i = tid; i < kSortChunk / 32 * kMaxE; i += kSortChunk) (&warp_at[0][0])[i] = 0;
  __syncthreads();
  {
    const int n_sub = kSortChunk / a.E, e = tid % a.E, sub = tid / a.E;
    if (sub < n_sub) {
      int all = 0, mine = 0;
      const int* c = a.counts + (size_t)l * a.B * a.E + e;
#pragma unroll 8
      for (int i = sub; i < a.B; i += n_sub) {
        const int n = c[(size_t)i * a.E];
        all += n;
        if (i < b) mine += n;
      }
      atomicAdd(&total[e], all);
      atomicAdd(&before[e], mine);
    }
  }
  __syncthreads();
  if (warp == 0) {   // exclusive scan over the experts
    int run = 0;
    for (int e0 = 0; e0 < a.E; e0 += 32) {
      const int n = e0 + lane < a.E ? total[e0 + lane] : 0;
      int s = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, s, o);
        if (lane >= o) s += v;
      }
      if (e0 + lane < a.E) {
        before[e0 + lane] += run + s - n;
        if (b == 0) a.offsets[(size_t)l * (a.E + 1) + e0 + lane] = run + s - n;
      }
      run += __shfl_sync(kFull, s, 31);
    }
    if (b == 0 && lane == 0) a.offsets[(size_t)l * (a.E + 1) + a.E] = run;
  }
  const int64_t q = (int64_t)b * kSortChunk + tid;
  int e = q < a.P ? a.sel[(size_t)l * a.P + q] : -1;
  if ((unsigned)e >= (unsigned)a.E) e = -1;
  const unsigned peers = __match_any_sync(kFull, e);
  const int rank = __popc(peers & ((1u << lane) - 1u));
  if (e >= 0 && rank == 0) warp_at[warp][e] = __popc(peers);
  __syncthreads();
  if (tid < a.E) {
    int run = before[tid];
    for (int w = 0; w < kSortChunk / 32; ++w) {
      const int n = warp_at[w][tid];
      warp_at[w][tid] = run;
      run += n;
    }
  }
  __syncthreads();
  if (q < a.P) {
    const int pos = e >= 0 ? warp_at[warp][e] + rank : -1;
    a.inv[(size_t)l * a.P + q] = pos;
    if (a.perm && pos >= 0) a.perm[(size_t)l * a.P + pos] = (int)q;
  }
}

struct CopyArgs {
  int64_t tokens;        // L * T
  int T, K, n_units, scale_cols;
  int64_t ld_x, ld_rows;   // in bytes
  const int32_t* inv;
  const char* x;
  char* rows;
  const float* scales;
  float* row_scales;
};

// A warp per token: its row is read once, a unit at a time, and written to the positions of its pairs.
template <typename V>
__global__ void __launch_bounds__(256) rows_copy_kernel(const CopyArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  const int64_t first = t / a.T * a.T * a.K;   // first sorted row of the token's layer
  const int my = lane < a.K ? a.inv[t * a.K + lane] : -1;
  const V* x = (const V*)(a.x + t * a.ld_x);
  for (int u = lane; u - lane < a.n_units; u += 32) {
    V v{};
    if (u < a.n_units) v = __ldg(x + u);
    for (int k = 0; k < a.K; ++k) {
      const int pos = __shfl_sync(kFull, my, k);
      if (pos >= 0 && u < a.n_units) ((V*)(a.rows + (first + pos) * a.ld_rows))[u] = v;
    }
  }
  for (int c = lane; c - lane < a.scale_cols; c += 32)
    for (int k = 0; k < a.K; ++k) {
      const int pos = __shfl_sync(kFull, my, k);
      if (pos >= 0 && c < a.scale_cols) a.row_scales[(first + pos) * a.scale_cols + c] = a.scales[t * a.scale_cols + c];
    }
}

struct CombineArgs {
  int64_t tokens, ld_token, ld_rows;
  int T, K, P, d;
  const int32_t* inv;
  const float* w;
  const void *rows, *add;
  void* y;
  const void* dy;
  void* drows;
  float* dw;
};

// A warp per token, U columns per lane at a time.
template <typename T, typename Y, int U>
__global__ void __launch_bounds__(256) combine_rows_kernel(const CombineArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  const T* rows = (const T*)a.rows + t / a.T * a.P * a.ld_rows;
  int my = lane < a.K ? a.inv[t * a.K + lane] : -1;
  if ((unsigned)my >= (unsigned)a.P) my = -1;
  const float my_w = lane < a.K && a.w ? a.w[t * a.K + lane] : 1.f;
  for (int c = lane * U; c - lane * U < a.d; c += 32 * U) {
    const bool in = c < a.d;
    float s[U];
#pragma unroll
    for (int i = 0; i < U; ++i) s[i] = 0.f;
    for (int k = 0; k < a.K; ++k) {
      const int pos = __shfl_sync(kFull, my, k);
      const float w = __shfl_sync(kFull, my_w, k);
      if (pos < 0 || !in) continue;
      Pack<T, U> p;
      p.load_const(rows + (int64_t)pos * a.ld_rows + c);
      float v[U];
      p.get(v);
#pragma unroll
      for (int i = 0; i < U; ++i) s[i] = fmaf(w, v[i], s[i]);
    }
    if (!in) continue;
    Pack<Y, U> y;
    if (a.add) {
      y.load((const Y*)a.add + t * a.ld_token + c);
      float v[U];
      y.get(v);
#pragma unroll
      for (int i = 0; i < U; ++i) s[i] += v[i];
    }
    y.set(s);
    y.store((Y*)a.y + t * a.ld_token + c);
  }
}

template <typename T, typename Y, int U>
__global__ void __launch_bounds__(256) combine_rows_grad_kernel(const CombineArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  const int64_t first = t / a.T * a.P;
  const Y* dy = (const Y*)a.dy + t * a.ld_token;
  for (int k = 0; k < a.K; ++k) {
    const int pos = a.inv[t * a.K + k];
    float dot = 0.f;
    if ((unsigned)pos < (unsigned)a.P) {
      const float w = a.w ? a.w[t * a.K + k] : 1.f;
      for (int c = lane * U; c < a.d; c += 32 * U) {
        Pack<Y, U> p;
        p.load_const(dy + c);
        float g[U], v[U];
        p.get(g);
        if (a.dw) {
          Pack<T, U> o;
          o.load((const T*)a.rows + (first + pos) * a.ld_rows + c);
          o.get(v);
#pragma unroll
          for (int i = 0; i < U; ++i) dot = fmaf(g[i], v[i], dot);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) v[i] = w * g[i];
        Pack<T, U> o;
        o.set(v);
        o.store((T*)a.drows + (first + pos) * a.ld_rows + c);
      }
    }
    if (a.dw) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(kFull, dot, o);
      if (lane == 0) a.dw[t * a.K + k] = dot;
    }
  }
}

struct UnitRule {
  int u;
  UnitRule(int d, int widest) : u(widest) {
    while (d % u) u /= 2;
  }
  void tensor(const void* p, int64_t ld, int elem_bytes) {
    while (p && u > 1) {
      const int a = u * elem_bytes > 16 ? 16 : u * elem_bytes;
      if ((uintptr_t)p % a == 0 && (ld * elem_bytes) % a == 0) return;
      u /= 2;
    }
  }
};

bool rows_ok(const mcce_rows* r) {
  if (!r) return false;
  if (r->n_layers < 1 || r->n_layers > 65535 || r->n_tokens < 0 || r->top_k < 1 || r->top_k > kMaxK || r->d < 1) return false;
  if ((int64_t)r->n_tokens * r->top_k > (1ll << 30)) return false;
  if ((r->ld_token && r->ld_token < r->d) || (r->ld_rows && r->ld_rows < r->d)) return false;
  return r->scale_cols >= 0;
}
bool dispatch_ok(const mcce_rows* r) {
  return rows_ok(r) && r->n_experts >= 1 && r->n_experts <= kMaxE && r->dtype >= MCCE_F32 && r->dtype <= MCCE_E4M3;
}
bool combine_ok(const mcce_rows* r) {
  return rows_ok(r) && (r->dtype == MCCE_F32 || r->dtype == MCCE_BF16) &&
         (r->token_dtype == MCCE_F32 || r->token_dtype == r->dtype);
}
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
int elem(int dtype) { return dtype == MCCE_F32 ? 4 : dtype == MCCE_BF16 ? 2 : 1; }
int64_t ld_or(int64_t ld, int d) { return ld ? ld : d; }

CombineArgs combine_args(const mcce_rows& r) {
  CombineArgs a{};
  a.tokens = (int64_t)r.n_layers * r.n_tokens, a.ld_token = ld_or(r.ld_token, r.d), a.ld_rows = ld_or(r.ld_rows, r.d);
  a.T = r.n_tokens, a.K = r.top_k, a.P = r.n_tokens * r.top_k, a.d = r.d;
  return a;
}

template <typename T, typename Y>
cudaError_t run_combine(const CombineArgs& a, int u, bool grad, cudaStream_t st) {
  const int64_t grid = (a.tokens + 7) / 8;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  auto go = [&](auto unit) {
    constexpr int U = decltype(unit)::value;
    if (grad) combine_rows_grad_kernel<T, Y, U><<<(unsigned)grid, 256, 0, st>>>(a);
    else combine_rows_kernel<T, Y, U><<<(unsigned)grid, 256, 0, st>>>(a);
  };
  if (u == 8) go(std::integral_constant<int, 8>{});
  else if (u == 4) go(std::integral_constant<int, 4>{});
  else if (u == 2) go(std::integral_constant<int, 2>{});
  else go(std::integral_constant<int, 1>{});
  return cudaGetLastError();
}
cudaError_t run_combine_any(const mcce_rows& r, const CombineArgs& a, int u, bool grad, cudaStream_t st) {
  if (r.dtype == MCCE_F32) return run_combine<float, float>(a, u, grad, st);
  if (r.token_dtype == MCCE_F32) return run_combine<__nv_bfloat16, float>(a, u, grad, st);
  return run_combine<__nv_bfloat16, __nv_bfloat16>(a, u, grad, st);
}

}  // namespace
}  // namespace mcce

using namespace mcce;

extern "C" size_t mcce_dispatch_workspace_bytes(const mcce_rows* r) {
  if (!dispatch_ok(r)) return 0;
  const size_t P = (size_t)r->n_tokens * r->top_k, B = (P + kSortChunk - 1) / kSortChunk;
  return (size_t)r->n_layers * B * r->n_experts * 4;
}

extern "C" int mcce_dispatch(const mcce_rows* r, const int32_t* sel_idx, const void* x, const float* scales,
                             int32_t* offsets, int32_t* perm, int32_t* inv, void* rows, float* row_scales,
                             void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!dispatch_ok(r) || !offsets || !aligned(offsets, 4)) return MCCE_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (r->n_tokens == 0)
    return cudaMemsetAsync(offsets, 0, (size_t)r->n_layers * (r->n_experts + 1) * 4, st) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
  if (!sel_idx || !inv) return MCCE_EINVAL;
  if ((x == nullptr) != (rows == nullptr)) return MCCE_EINVAL;
  const bool with_scales = r->scale_cols > 0;
  if (with_scales != (scales != nullptr) || with_scales != (row_scales != nullptr)) return MCCE_EINVAL;
  const int e = elem(r->dtype);
  if (!aligned(x, e) || !aligned(rows, e) || !aligned(scales, 4) || !aligned(row_scales, 4) || !aligned(sel_idx, 4) ||
      !aligned(perm, 4) || !aligned(inv, 4))
    return MCCE_EINVAL;
  const size_t need = mcce_dispatch_workspace_bytes(r);
  if (need && (!workspace || !aligned(workspace, 16))) return MCCE_EINVAL;
  if (workspace_bytes < need) return MCCE_ENOSPC;
  SortArgs s;
  s.T = r->n_tokens, s.K = r->top_k, s.E = r->n_experts, s.P = s.T * s.K, s.B = (s.P + kSortChunk - 1) / kSortChunk;
  s.sel = sel_idx, s.offsets = offsets, s.perm = perm, s.inv = inv, s.counts = (int32_t*)workspace;
  const dim3 grid(s.B, r->n_layers);
  rows_count_kernel<<<grid, 256, 0, st>>>(s);
  rows_rank_kernel<<<grid, kSortChunk, 0, st>>>(s);
  if (x || with_scales) {
    CopyArgs c;
    c.tokens = (int64_t)r->n_layers * r->n_tokens, c.T = s.T, c.K = s.K, c.scale_cols = r->scale_cols;
    c.ld_x = ld_or(r->ld_token, r->d) * e, c.ld_rows = ld_or(r->ld_rows, r->d) * e;
    c.inv = inv, c.x = (const char*)x, c.rows = (char*)rows, c.scales = scales, c.row_scales = row_scales;
    const int64_t bytes = x ? (int64_t)r->d * e : 0;
    int v = 16;
    while (v > 1 && (bytes % v || c.ld_x % v || c.ld_rows % v || !aligned(x, v) || !aligned(rows, v))) v /= 2;
    c.n_units = (int)(bytes / v);
    const int64_t g = (c.tokens + 7) / 8;
    if (g > 0x7fffffffll) return MCCE_EINVAL;
    if (v == 16) rows_copy_kernel<uint4><<<(unsigned)g, 256, 0, st>>>(c);
    else if (v == 8) rows_copy_kernel<uint2><<<(unsigned)g, 256, 0, st>>>(c);
    else if (v == 4) rows_copy_kernel<uint32_t><<<(unsigned)g, 256, 0, st>>>(c);
    else if (v == 2) rows_copy_kernel<uint16_t><<<(unsigned)g, 256, 0, st>>>(c);
    else rows_copy_kernel<uint8_t><<<(unsigned)g, 256, 0, st>>>(c);
  }
  return cudaGetLastError() == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}

extern "C" int mcce_combine(const mcce_rows* r, const void* rows, const int32_t* inv, const float* sel_w,
                            const void* add, void* y, void* cuda_stream) {
  if (!combine_ok(r)) return MCCE_EINVAL;
  if (r->n_tokens == 0) return MCCE_OK;
  if (!rows || !inv || !y) return MCCE_EINVAL;
  const int e = elem(r->dtype), ey = elem(r->token_dtype);
  if (!aligned(rows, e) || !aligned(inv, 4) || !aligned(sel_w, 4) || !aligned(add, ey) || !aligned(y, ey)) return MCCE_EINVAL;
  CombineArgs a = combine_args(*r);
  a.inv = inv, a.w = sel_w, a.rows = rows, a.add = add, a.y = y;
  UnitRule u(r->d, 8);
  u.tensor(rows, a.ld_rows, e);
  u.tensor(add, a.ld_token, ey);
  u.tensor(y, a.ld_token, ey);
  return run_combine_any(*r, a, u.u, false, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}

extern "C" int mcce_combine_backward(const mcce_rows* r, const void* dy, const void* rows, const int32_t* inv,
                                     const float* sel_w, void* drows, float* dw, void* cuda_stream) {
  if (!combine_ok(r)) return MCCE_EINVAL;
  if (r->n_tokens == 0) return MCCE_OK;
  if (!dy || !inv || !drows || (dw && !rows)) return MCCE_EINVAL;
  const int e = elem(r->dtype), ey = elem(r->token_dtype);
  if (!aligned(rows, e) || !aligned(drows, e) || !aligned(inv, 4) || !aligned(sel_w, 4) || !aligned(dy, ey) || !aligned(dw, 4))
    return MCCE_EINVAL;
  CombineArgs a = combine_args(*r);
  a.inv = inv, a.w = sel_w, a.rows = rows, a.dy = dy, a.drows = drows, a.dw = dw;
  UnitRule u(r->d, 8);
  u.tensor(dw ? rows : nullptr, a.ld_rows, e);
  u.tensor(drows, a.ld_rows, e);
  u.tensor(dy, a.ld_token, ey);
  return run_combine_any(*r, a, u.u, true, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
