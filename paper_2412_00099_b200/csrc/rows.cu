// Token rows sorted by expert, the rows brought back to their tokens with weights (Eq. 1's sum), and its gradient.
#include <type_traits>

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
  cudaGridDependencySynchronize();
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

// ---- moving rows ------------------------------------------------------------------------------------------------
// tpt threads per token (a power of two, 16 .. 256); a token's pairs are looked at by its first top_k threads and
// handed round the warp.
struct Token {
  int64_t t, first;   // token over all layers; first sorted row of its layer
  int lane0;          // first lane of the token in this warp
  int u0;             // this thread's index in the token
  bool there;
  __device__ __forceinline__ Token(int tpt, int64_t tokens, int T, int P) {
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    t = at / tpt;
    u0 = (int)at & (tpt - 1);
    lane0 = tpt < 32 ? (int)(threadIdx.x & 31) & ~(tpt - 1) : 0;
    there = t < tokens;
    first = there ? t / T * P : 0;
  }
};
// The position of pair k of a token, -1: none.  `mine` is the position of this lane's pair.
__device__ __forceinline__ int position(const Token& tk, int mine, int k) { return __shfl_sync(kFull, mine, tk.lane0 + k); }
__device__ __forceinline__ int my_position(const Token& tk, const int32_t* inv, int K, int P) {
  const int k = (int)(threadIdx.x & 31) - tk.lane0;
  const int pos = tk.there && k < K ? inv[tk.t * K + k] : -1;
  return (unsigned)pos < (unsigned)P ? pos : -1;
}

struct CopyArgs {
  int64_t tokens;        // L * T
  int64_t ld_x, ld_rows; // in units
  int T, K, P, units, scale_cols, tpt;
  const int32_t* inv;
  const void* x;
  void* rows;
  const float* scales;
  float* row_scales;
};

// The row of a token to the positions of its pairs, by `threads` threads of which this is number u0.  V units of the row are
// read, all in flight, and written once for every pair: a token's row is read once.
// position_of(k): of pair k, -1: none.
template <typename V_, typename F>
__device__ __forceinline__ void move_row(const CopyArgs& a, int64_t t, int64_t first, int u0, int threads, F position_of) {
  constexpr int V = sizeof(V_) == 16 ? 4 : 8;
  const V_* x = (const V_*)a.x + t * a.ld_x;
  V_* rows = (V_*)a.rows + first * a.ld_rows;
  for (int b = u0; b - u0 < a.units; b += threads * V) {
    V_ p[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (b + v * threads < a.units) p[v] = __ldg(x + b + v * threads);
    for (int k = 0; k < a.K; ++k) {
      const int pos = position_of(k);
      if (pos < 0) continue;
      V_* to = rows + pos * a.ld_rows + b;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (b + v * threads < a.units) to[v * threads] = p[v];
    }
  }
}

template <typename V>
__global__ void __launch_bounds__(256) rows_copy_kernel(const __grid_constant__ CopyArgs a) {
  cudaGridDependencySynchronize();
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  if (a.x) move_row<V>(a, tk.there ? tk.t : 0, tk.first, tk.u0, a.tpt, [&](int k) { return position(tk, mine, k); });
  for (int k = 0; a.scale_cols && k < a.K; ++k) {
    const int pos = position(tk, mine, k);
    for (int c = tk.u0; pos >= 0 && c < a.scale_cols; c += a.tpt)
      a.row_scales[(tk.first + pos) * a.scale_cols + c] = a.scales[tk.t * a.scale_cols + c];
  }
}

// Few pairs per layer: one launch.  Every CTA counts all pairs of its layer (and, in the upper half of a word, those before
// its own tokens), ranks its own and moves their rows; the counting takes the place of two more launches.
constexpr int kFusedPairs = 64;    // pairs of a CTA at most
template <typename V>
__global__ void __launch_bounds__(256) rows_dispatch_kernel(const __grid_constant__ SortArgs s, const __grid_constant__ CopyArgs a,
                                                            const int tokens_per_cta) {
  __shared__ int count[kMaxE], base[kMaxE], warp_sum[8], id[kFusedPairs], place[kFusedPairs];
  const int l = blockIdx.y, t0 = blockIdx.x * tokens_per_cta, n_tok = min(tokens_per_cta, s.T - t0);
  const int q0 = t0 * s.K, n = n_tok * s.K, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t* sel = s.sel + (size_t)l * s.P;
  count[tid] = 0;
  __syncthreads();
  if (tid < n) {
    const int e = sel[q0 + tid];
    id[tid] = (unsigned)e < (unsigned)s.E ? e : -1;
  }
#pragma unroll 4
  for (int q = tid; q < s.P; q += 256) {
    const int e = sel[q];
    if ((unsigned)e < (unsigned)s.E) atomicAdd(&count[e], q < q0 ? 0x10001 : 1);
  }
  __syncthreads();
  const int c = count[tid], all = c & 0xffff;
  int run = all;   // inclusive scan over the experts
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(kFull, run, o);
    if (lane >= o) run += v;
  }
  if (lane == 31) warp_sum[warp] = run;
  __syncthreads();
  for (int w = 0; w < warp; ++w) run += warp_sum[w];
  base[tid] = run - all + (c >> 16);
  if (blockIdx.x == 0) {
    int32_t* off = s.offsets + (size_t)l * (s.E + 1);
    if (tid < s.E) off[tid + 1] = run;
    if (tid == 0) off[0] = 0;
  }
  __syncthreads();
  if (tid < n) {
    const int e = id[tid];
    int pos = -1;
    if (e >= 0) {
      pos = base[e];
      for (int j = 0; j < tid; ++j) pos += id[j] == e;
    }
    place[tid] = pos;
    s.inv[(size_t)l * s.P + q0 + tid] = pos;
    if (s.perm && pos >= 0) s.perm[(size_t)l * s.P + pos] = q0 + tid;
  }
  __syncthreads();
  // the warps of a token: one each for eight tokens or more, else the eight warps shared out
  const int64_t first = (int64_t)l * s.P;
  const int per_token = n_tok >= 8 ? 1 : n_tok >= 4 ? 2 : n_tok >= 2 ? 4 : 8, slots = 8 / per_token;
  const int u0 = (warp & (per_token - 1)) * 32 + lane;
  for (int t = warp / per_token; t < n_tok; t += slots) {
    const int64_t token = (int64_t)l * s.T + t0 + t;
    if (a.x) move_row<V>(a, token, first, u0, per_token * 32, [&](int k) { return place[t * s.K + k]; });
    for (int k = 0; a.scale_cols && k < s.K; ++k) {
      const int pos = place[t * s.K + k];
      for (int i = u0; pos >= 0 && i < a.scale_cols; i += per_token * 32)
        a.row_scales[(first + pos) * a.scale_cols + i] = a.scales[token * a.scale_cols + i];
    }
  }
}

struct CombineArgs {
  int64_t tokens, ld_token, ld_rows;
  int T, K, P, d, tpt;
  const int32_t* inv;
  const float* w;
  const void *rows, *add;
  void* y;
  const void* dy;
  void* drows;
  float* dw;
};

// y of a token: U columns at a time, VPT such units per thread and KC rows at once, so that KC * VPT loads are in flight.
template <typename T, typename Y, int U, int KC, int VPT>
__global__ void __launch_bounds__(256) combine_rows_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int N = (U + 1) / 2;
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  const float my_w = mine >= 0 && a.w ? a.w[tk.t * a.K + (int)(threadIdx.x & 31) - tk.lane0] : 1.f;
  const T* rows = (const T*)a.rows + tk.first * a.ld_rows;
  const int64_t at = tk.t * a.ld_token;
  const int d = tk.there ? a.d : 0, step = a.tpt * U;
  for (int b = 0; b < a.d; b += step * VPT) {
    const int c0 = b + tk.u0 * U;
    float2 s[VPT][N];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int j = 0; j < N; ++j) s[v][j] = both(0.f);
    for (int k0 = 0; k0 < a.K; k0 += KC) {
      Pack<T, U> p[KC][VPT];
      float w[KC];
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const int pos = k0 + k < a.K ? position(tk, mine, k0 + k) : -1;
        w[k] = __shfl_sync(kFull, my_w, tk.lane0 + ((k0 + k) & 15));
        const T* row = rows + pos * a.ld_rows + c0;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          p[k][v].zero();
          if (pos >= 0 && c0 + v * step < d) p[k][v].load_const(row + v * step);
        }
      }
#pragma unroll
      for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          float2 e[N];
          p[k][v].get(e);
#pragma unroll
          for (int j = 0; j < N; ++j) s[v][j] = fma2(e[j], both(w[k]), s[v][j]);
        }
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = c0 + v * step;
      if (c >= d) continue;
      Pack<Y, U> y;
      if (a.add) {
        y.load((const Y*)a.add + at + c);
        float2 e[N];
        y.get(e);
#pragma unroll
        for (int j = 0; j < N; ++j) s[v][j] = add2(s[v][j], e[j]);
      }
      y.set(s[v]);
      y.store((Y*)a.y + at + c);
    }
  }
}

// Sums of acc[k] over `lanes` lanes, k < KC.  The number of values is halved while the lanes that share one double, so KC sums
// cost little more than one; lane l holds that of k = l / (lanes / KC) afterwards.
template <int KC>
__device__ __forceinline__ float sum_of_all(float (&acc)[KC], int lanes) {
  int o = lanes >> 1;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = KC / 2; n > 0; n >>= 1, o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float keep = upper ? acc[n + k] : acc[k], give = upper ? acc[k] : acc[n + k];
      acc[k] = keep + __shfl_xor_sync(kFull, give, o);
    }
  }
  for (; o > 0; o >>= 1) acc[0] += __shfl_xor_sync(kFull, acc[0], o);
  return acc[0];
}

// drows and dw of a token: a unit of a row is read, multiplied into the pair's sum, and replaced by w dy.  KC rows at once.
template <typename T, typename Y, int U, int KC, int VPT>
__global__ void __launch_bounds__(256) combine_rows_grad_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int N = (U + 1) / 2;
  __shared__ float parts[8][KC];
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  const float my_w = mine >= 0 && a.w ? a.w[tk.t * a.K + (int)(threadIdx.x & 31) - tk.lane0] : 1.f;
  const T* rows = (const T*)a.rows;
  T* drows = (T*)a.drows;
  const Y* dy = (const Y*)a.dy + tk.t * a.ld_token;
  const int d = tk.there ? a.d : 0, step = a.tpt * U;
  for (int k0 = 0; k0 < a.K; k0 += KC) {
    int64_t at[KC];   // first element of the pair's row, -1: no row
    float w[KC], acc[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const int pos = k0 + k < a.K ? position(tk, mine, k0 + k) : -1;
      w[k] = __shfl_sync(kFull, my_w, tk.lane0 + ((k0 + k) & 15));
      at[k] = pos >= 0 ? (tk.first + pos) * a.ld_rows : -1;
      acc[k] = 0.f;
    }
    for (int c = tk.u0 * U; c < d; c += step * VPT) {
      Pack<T, U> p[KC][VPT];
      Pack<Y, U> q[VPT];
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        if (c + v * step < d) q[v].load_const(dy + c + v * step);
      if (a.dw) {
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
          for (int v = 0; v < VPT; ++v)
            if (at[k] >= 0 && c + v * step < d) p[k][v].load(rows + at[k] + c + v * step);
      }
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        if (c + v * step >= d) continue;
        float2 g[N];
        q[v].get(g);
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          if (at[k] < 0) continue;
          float2 e[N];
          if (a.dw) {
            p[k][v].get(e);
            float2 s = both(0.f);
#pragma unroll
            for (int j = 0; j < N; ++j) s = fma2(e[j], g[j], s);
            acc[k] += s.x + s.y;
          }
#pragma unroll
          for (int j = 0; j < N; ++j) e[j] = mul2(g[j], both(w[k]));
          p[k][v].set(e);
          p[k][v].store(drows + at[k] + c + v * step);
        }
      }
    }
    if (!a.dw) continue;
    const int lane = threadIdx.x & 31, lanes = min(a.tpt, 32);
    const float s = sum_of_all(acc, lanes);
    const int k = (lane & (lanes - 1)) / (lanes / KC);
    const bool speaks = (lane & (lanes / KC - 1)) == 0;
    if (a.tpt <= 32) {
      if (speaks && tk.there && k0 + k < a.K) a.dw[tk.t * a.K + k0 + k] = s;
    } else {
      __syncthreads();   // the last chunk's parts have been read
      if (speaks) parts[threadIdx.x >> 5][k] = s;
      __syncthreads();
      if (tk.there && tk.u0 < KC && k0 + tk.u0 < a.K) {
        const int warps = a.tpt >> 5, w0 = threadIdx.x >> 5;
        float v = 0.f;
        for (int i = 0; i < warps; ++i) v += parts[w0 + i][tk.u0];
        a.dw[tk.t * a.K + k0 + tk.u0] = v;
      }
    }
  }
}

// Host: the widest unit (at most `widest` elements, a power of two) that divides the width and for which every row of every
// tensor starts aligned.
struct UnitRule {
  int u;
  UnitRule(int d, int widest) : u(widest) {
    while (d % u) u /= 2;
  }
  void tensor(const void* p, int64_t ld, int elem_bytes) {   // null: not part of the call
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

// Threads per token: a power of two that covers the row's units `per_thread` at a time, within 16 .. 256.
int threads_per_token(int units, int per_thread) {
  int t = 16;
  while (t < 256 && t * per_thread < units) t *= 2;
  return t;
}
template <typename K>
cudaError_t launch_tokens(K kernel, const CombineArgs& a, cudaStream_t st) {
  const int64_t grid = (a.tokens * a.tpt + 255) / 256;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  kernel<<<(unsigned)grid, 256, 0, st>>>(a);
  return cudaGetLastError();
}

// Many tokens: a few units per thread.  Few tokens: one.
int spread(const CombineArgs& a, int u, int units_per_thread) {
  return threads_per_token((a.d + u - 1) / u, a.tokens * 64 < 148 * 1024 ? 1 : units_per_thread);
}

// Rows at once x units at once and threads per token, us measured (one launch between two events, 5 us of it not the kernel's;
// 16384 tokens of 2048 bf16 columns unless noted).  Return, K = 8: 4 x 1 on 64 threads 99 (0.93 of the copy bandwidth), 8 x 1 104,
// 2 x 2 133; K = 2, 4099 tokens of 4096: 1 x 4 22.8, 2 x 2 24.1, 2 x 1 25.2; K = 1 of 4096: 1 x 4 47.8, 2 x 2 55.7.  Gradient, K = 8:
// 2 x 2 on 32 threads 195 (0.89), 4 x 1 193, 1 x 2 222; K = 6: 151 / 163 / 156.
// Units narrower than 16 bytes (odd widths, unaligned rows) keep fewer bytes in flight per register: 8192 tokens, K = 8, of 1411
// columns: return 4 x 4 82 (0.39), 4 x 2 93; gradient 4 x 1 142 (0.42), 2 x 4 152.  Sixteen-byte loads at the next boundary, shifted
// into place, were no faster (74 .. 80 and 166).
template <typename T, typename Y, int U>
cudaError_t run_combine(CombineArgs a, cudaStream_t st) {
  if constexpr (U * sizeof(T) == 16) {
    a.tpt = spread(a, U, a.K <= 2 ? 8 : 4);
    if (a.K <= 2) return launch_tokens(combine_rows_kernel<T, Y, U, 1, 4>, a, st);
    return launch_tokens(combine_rows_kernel<T, Y, U, 4, sizeof(T) == 4 ? 2 : 1>, a, st);
  } else {
    a.tpt = spread(a, U, 32);
    if (a.K <= 2) return launch_tokens(combine_rows_kernel<T, Y, U, 1, 8>, a, st);
    return launch_tokens(combine_rows_kernel<T, Y, U, 4, 4>, a, st);
  }
}
template <typename T, typename Y, int U>
cudaError_t run_combine_grad(CombineArgs a, cudaStream_t st) {
  if constexpr (U * sizeof(T) == 16) {
    a.tpt = spread(a, U, 8);
    if (a.K == 1) return launch_tokens(combine_rows_grad_kernel<T, Y, U, 1, 2>, a, st);
    return launch_tokens(combine_rows_grad_kernel<T, Y, U, 2, 2>, a, st);
  } else {
    a.tpt = spread(a, U, a.K <= 2 ? 32 : 16);
    if (a.K <= 2) return launch_tokens(combine_rows_grad_kernel<T, Y, U, 2, 4>, a, st);
    return launch_tokens(combine_rows_grad_kernel<T, Y, U, 4, 1>, a, st);
  }
}
template <typename T, typename Y>
cudaError_t run_combine_unit(const CombineArgs& a, int u, bool grad, cudaStream_t st) {
  constexpr int kWide = 16 / (int)sizeof(T);
  if (u == kWide) return grad ? run_combine_grad<T, Y, kWide>(a, st) : run_combine<T, Y, kWide>(a, st);
  if (u >= 2) return grad ? run_combine_grad<T, Y, 2>(a, st) : run_combine<T, Y, 2>(a, st);
  return grad ? run_combine_grad<T, Y, 1>(a, st) : run_combine<T, Y, 1>(a, st);
}
cudaError_t run_combine_types(const mcce_rows& r, const CombineArgs& a, int u, bool grad, cudaStream_t st) {
  if (r.dtype == MCCE_F32) return run_combine_unit<float, float>(a, u, grad, st);
  if (r.token_dtype == MCCE_F32) return run_combine_unit<__nv_bfloat16, float>(a, u, grad, st);
  return run_combine_unit<__nv_bfloat16, __nv_bfloat16>(a, u, grad, st);
}

// A launch that may begin while the kernel before it ends; the kernel waits for that one itself.
template <typename P>
cudaError_t launch_after(void (*kernel)(P), dim3 grid, int threads, cudaStream_t st, const std::decay_t<P>& args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.stream = st, cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args);
}

// Tokens per CTA of the single launch, 0: several launches.
int fused_tokens(const SortArgs& s) {
  if (s.P > 8192) return 0;
  return s.K >= 4 ? 4 : s.K >= 2 ? 8 : 16;
}

template <typename V>
cudaError_t run_dispatch(const SortArgs& s, CopyArgs c, int L, cudaStream_t st) {
  if (const int t = fused_tokens(s)) {
    rows_dispatch_kernel<V><<<dim3((s.T + t - 1) / t, L), 256, 0, st>>>(s, c, t);
    return cudaGetLastError();
  }
  const dim3 grid(s.B, L);
  rows_count_kernel<<<grid, 256, 0, st>>>(s);
  cudaError_t err = cudaGetLastError();
  if (err == cudaSuccess) err = launch_after(rows_rank_kernel, grid, kSortChunk, st, s);
  if (err != cudaSuccess || !(c.x || c.scale_cols)) return err;
  c.tpt = threads_per_token(c.units, sizeof(V) == 16 ? 2 : 16);
  if (c.tpt > 128) c.tpt = 128;
  const int64_t ctas = (c.tokens * c.tpt + 255) / 256;
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_after(rows_copy_kernel<V>, dim3((unsigned)ctas), 256, st, c);
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
  CopyArgs c{};
  c.tokens = (int64_t)r->n_layers * r->n_tokens, c.T = s.T, c.K = s.K, c.P = s.P, c.scale_cols = r->scale_cols;
  c.inv = inv, c.x = x, c.rows = rows, c.scales = scales, c.row_scales = row_scales;
  // rows are moved in units of 16 bytes or the largest power of two that they are aligned to
  int64_t ld_x = ld_or(r->ld_token, r->d) * e, ld_rows = ld_or(r->ld_rows, r->d) * e, row = x ? (int64_t)r->d * e : 0;
  int v = 16;
  while (v > 1 && (row % v || ld_x % v || ld_rows % v || !aligned(x, v) || !aligned(rows, v))) v /= 2;
  c.ld_x = ld_x / v, c.ld_rows = ld_rows / v, c.units = (int)(row / v);
  cudaError_t err;
  if (v == 16) err = run_dispatch<uint4>(s, c, r->n_layers, st);
  else if (v == 8) err = run_dispatch<uint2>(s, c, r->n_layers, st);
  else if (v == 4) err = run_dispatch<uint32_t>(s, c, r->n_layers, st);
  else if (v == 2) err = run_dispatch<uint16_t>(s, c, r->n_layers, st);
  else err = run_dispatch<uint8_t>(s, c, r->n_layers, st);
  return err == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
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
  UnitRule u(r->d, 16 / e);
  u.tensor(rows, a.ld_rows, e);
  u.tensor(add, a.ld_token, ey);
  u.tensor(y, a.ld_token, ey);
  return run_combine_types(*r, a, u.u, false, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
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
  a.inv = inv, a.w = sel_w, a.rows = dw ? rows : nullptr, a.dy = dy, a.drows = drows, a.dw = dw;
  UnitRule u(r->d, 16 / e);
  u.tensor(a.rows, a.ld_rows, e);
  u.tensor(drows, a.ld_rows, e);
  u.tensor(dy, a.ld_token, ey);
  return run_combine_types(*r, a, u.u, true, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
