// Token rows sorted by expert, the rows brought back to their tokens with weights (Eq. 1's sum), and its gradient.
#include <type_traits>

#include "common.cuh"
#include "vec.cuh"

namespace mcce {
namespace {

constexpr unsigned kFull = 0xffffffffu;
struct SortArgs {
  int T, K, E, P;
  int chunk, B;   // tokens per chunk, chunks per layer
  const int32_t* sel;
  int32_t *offsets, *perm, *inv, *counts;   // counts [L][B][E], not used when B is 1
};

// Pairs of every expert in a chunk of a layer.
__global__ void __launch_bounds__(256) rows_count_kernel(const __grid_constant__ SortArgs s) {
  __shared__ int count[kMaxE];
  const int b = blockIdx.x, l = blockIdx.y;
  count[threadIdx.x] = 0;
  __syncthreads();
  const int32_t* sel = s.sel + (size_t)l * s.P;
  const int end = min(s.P, (b + 1) * s.chunk * s.K);
#pragma unroll 4
  for (int q = b * s.chunk * s.K + threadIdx.x; q < end; q += 256) {
    const int e = sel[q];
    if ((unsigned)e < (unsigned)s.E) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  if ((int)threadIdx.x < s.E) s.counts[((size_t)l * s.B + b) * s.E + threadIdx.x] = count[threadIdx.x];
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
  int64_t ld_x, ld_rows; // in units
  int K, units, scale_cols;
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

// Ranks the pairs of a few tokens and moves their rows.  Where a pair goes: pairs of smaller experts (totals of all chunks), of
// its expert in earlier chunks (both from the chunks' counts), earlier in its chunk (counted here again), earlier in this
// CTA.  A layer of few pairs is one chunk: the CTA counts all of it, and there is no launch before this one.
constexpr int kCtaPairs = 128;    // pairs of a CTA at most
template <typename V>
__global__ void __launch_bounds__(256) rows_dispatch_kernel(const __grid_constant__ SortArgs s, const __grid_constant__ CopyArgs a,
                                                            const int tokens_per_cta) {
  __shared__ int total[kMaxE], before[kMaxE], warp_sum[8], id[kCtaPairs], place[kCtaPairs];
  const int l = blockIdx.y, t0 = blockIdx.x * tokens_per_cta, n_tok = min(tokens_per_cta, s.T - t0);
  const int q0 = t0 * s.K, n = n_tok * s.K, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = t0 / s.chunk, chunk0 = b * s.chunk * s.K;
  const int32_t* sel = s.sel + (size_t)l * s.P;
  total[tid] = before[tid] = 0;
  __syncthreads();
  if (tid < n) {
    const int e = sel[q0 + tid];
    id[tid] = (unsigned)e < (unsigned)s.E ? e : -1;
  }
  if (s.B == 1) {   // total and, in the upper half of a word, before
#pragma unroll 4
    for (int q = tid; q < s.P; q += 256) {
      const int e = sel[q];
      if ((unsigned)e < (unsigned)s.E) atomicAdd(&total[e], q < q0 ? 0x10001 : 1);
    }
  } else {
#pragma unroll 4
    for (int q = chunk0 + tid; q < q0; q += 256) {
      const int e = sel[q];
      if ((unsigned)e < (unsigned)s.E) atomicAdd(&before[e], 1);
    }
    cudaGridDependencySynchronize();
    const int n_sub = 256 / s.E, e = tid % s.E, sub = tid / s.E;
    if (sub < n_sub) {
      const int32_t* c = s.counts + (size_t)l * s.B * s.E + e;
      int all = 0, mine = 0;
#pragma unroll 8
      for (int i = sub; i < s.B; i += n_sub) {
        const int v = c[(size_t)i * s.E];
        all += v;
        if (i < b) mine += v;
      }
      atomicAdd(&total[e], all);
      atomicAdd(&before[e], mine);
    }
  }
  __syncthreads();
  const int packed = total[tid], all = s.B == 1 ? packed & 0xffff : packed;
  int run = all;   // inclusive scan over the experts
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(kFull, run, o);
    if (lane >= o) run += v;
  }
  if (lane == 31) warp_sum[warp] = run;
  __syncthreads();
  for (int w = 0; w < warp; ++w) run += warp_sum[w];
  before[tid] += run - all + (s.B == 1 ? packed >> 16 : 0);
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
      pos = before[e];
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

// How the pairs of a layer are split: tokens per CTA (`cta`), tokens per chunk (a multiple of it) and chunks.
struct SortShape {
  int cta, chunk, B;
};
// A CTA moves up to 160 KB: 16384 tokens x 8 of 2048 bytes with scales, us, 4 / 8 tokens: 63.6 / 59; of 4096 bytes 2 / 4 / 8 tokens:
// 106 / 109 / 111; 24 x 256 tokens x 4 of 4096 bytes 27 / 25 / 27.  Chunks of 2048 pairs: between 512 and 4096 the time changes by
// 1 %.  A layer is one chunk -- one launch, every CTA counts the whole layer -- while that is little work: 24 x 256 tokens x 4
// 25.0 against 27.9 with two launches, 4096 tokens x 2 of 8192 bytes 32.7 against 22.8.
SortShape sort_shape(const mcce_rows& r) {
  const int K = r.top_k, T = r.n_tokens;
  const int64_t moved = (int64_t)(K + 1) * r.d * (r.dtype == MCCE_F32 ? 4 : r.dtype == MCCE_BF16 ? 2 : 1);
  SortShape h;
  h.cta = 1;
  while (h.cta * 2 * K <= kCtaPairs && h.cta * 2 * moved <= 160 * 1024) h.cta *= 2;
  const int64_t pairs = (int64_t)T * K, ctas = (int64_t)r.n_layers * ((T + h.cta - 1) / h.cta);
  if (pairs <= 2048 || (pairs <= 8192 && ctas * pairs <= (2 << 20))) {
    h.chunk = T, h.B = 1;
    return h;
  }
  const int most = 16384 / r.n_experts < 256 ? 16384 / r.n_experts : 256;   // chunks: every CTA reads all counts
  int chunk = 2048 / K;
  if ((T + chunk - 1) / chunk > most) chunk = (T + most - 1) / most;
  h.chunk = (chunk + h.cta - 1) / h.cta * h.cta;
  h.B = (T + h.chunk - 1) / h.chunk;
  return h;
}

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

// With fewer tokens than this the device is not full: one unit per thread and as many threads per token as that takes.
bool few(const CombineArgs& a) { return a.tokens * 64 < 148 * 1024; }

// KC rows at once x VPT units at once, us measured back to back on rotating buffers (16384 tokens of 2048 bf16 columns unless
// noted).  Return, K = 8: 4 x 1 on 32 threads per token 96.6 (0.95 of the copy bandwidth), 8 x 1 104, 2 x 2 133; K = 2, 4099
// tokens of 4096: 2 x 4 22.7 (0.68), 1 x 4 24.5, 4 x 1 25; K = 1 of 4096: 1 x 4 45 (0.91), 2 x 2 56; 256 tokens, K = 8: 4 x 1 on 256 threads
// 4.2, 4 x 2 4.7.  Gradient, K = 8: 1 x 4 on 32 threads 188 (0.92), 4 x 1 191, 2 x 2 192; K = 1 of 4096: 1 x 4 66 (0.93); 256 tokens,
// K = 8: 4 x 1 on 256 threads 6.3, 2 x 2 8.3.
// Units narrower than 16 bytes (odd widths, unaligned rows) keep fewer bytes in flight per register: 8192 tokens, K = 8, of 1411
// bf16 columns: return 4 x 4 80 (0.40), 8 x 2 88; gradient 4 x 1 143 (0.42), 2 x 4 152.  Sixteen-byte loads at the next boundary, shifted
// into place, were no faster (74 .. 80 and 166).
template <typename T, typename Y, int U>
cudaError_t run_combine(CombineArgs a, cudaStream_t st) {
  constexpr bool kWide = U * sizeof(T) == 16;
  a.tpt = threads_per_token((a.d + U - 1) / U, few(a) ? 1 : kWide ? 8 : 32);
  if constexpr (kWide) {
    if (a.K == 1) return launch_tokens(combine_rows_kernel<T, Y, U, 1, 4>, a, st);
    if (a.K == 2) return launch_tokens(combine_rows_kernel<T, Y, U, 2, 4>, a, st);
    return launch_tokens(combine_rows_kernel<T, Y, U, 4, sizeof(T) == 4 ? 2 : 1>, a, st);
  } else {
    if (a.K <= 2) return launch_tokens(combine_rows_kernel<T, Y, U, 2, 4>, a, st);
    return launch_tokens(combine_rows_kernel<T, Y, U, 4, 4>, a, st);
  }
}
template <typename T, typename Y, int U>
cudaError_t run_combine_grad(CombineArgs a, cudaStream_t st) {
  constexpr bool kWide = U * sizeof(T) == 16;
  a.tpt = threads_per_token((a.d + U - 1) / U, few(a) ? 1 : kWide ? 8 : a.K <= 2 ? 32 : 16);
  if constexpr (kWide) {
    if (!few(a)) return launch_tokens(combine_rows_grad_kernel<T, Y, U, 1, 4>, a, st);
  } else {
    if (a.K <= 2) return launch_tokens(combine_rows_grad_kernel<T, Y, U, 2, 4>, a, st);
  }
  return launch_tokens(combine_rows_grad_kernel<T, Y, U, 4, 1>, a, st);
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
template <typename... P>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t st, const std::decay_t<P>&... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.stream = st, cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename V>
cudaError_t run_dispatch(const SortArgs& s, const CopyArgs& c, int L, int t, cudaStream_t st) {
  const dim3 grid((s.T + t - 1) / t, L);
  if (s.B == 1) {
    rows_dispatch_kernel<V><<<grid, 256, 0, st>>>(s, c, t);
    return cudaGetLastError();
  }
  rows_count_kernel<<<dim3(s.B, L), 256, 0, st>>>(s);
  const cudaError_t err = cudaGetLastError();
  return err == cudaSuccess ? launch_after(rows_dispatch_kernel<V>, grid, 256, st, s, c, t) : err;
}

}  // namespace
}  // namespace mcce

using namespace mcce;

extern "C" size_t mcce_dispatch_workspace_bytes(const mcce_rows* r) {
  if (!dispatch_ok(r)) return 0;
  if (r->n_tokens == 0) return 0;
  const SortShape h = sort_shape(*r);
  return h.B == 1 ? 0 : (size_t)r->n_layers * h.B * r->n_experts * 4;
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
  const SortShape h = sort_shape(*r);
  SortArgs s;
  s.T = r->n_tokens, s.K = r->top_k, s.E = r->n_experts, s.P = s.T * s.K, s.chunk = h.chunk, s.B = h.B;
  s.sel = sel_idx, s.offsets = offsets, s.perm = perm, s.inv = inv, s.counts = (int32_t*)workspace;
  CopyArgs c{};
  c.K = s.K, c.scale_cols = r->scale_cols;
  c.x = x, c.rows = rows, c.scales = scales, c.row_scales = row_scales;
  // rows are moved in units of 16 bytes or the largest power of two that they are aligned to
  int64_t ld_x = ld_or(r->ld_token, r->d) * e, ld_rows = ld_or(r->ld_rows, r->d) * e, row = x ? (int64_t)r->d * e : 0;
  int v = 16;
  while (v > 1 && (row % v || ld_x % v || ld_rows % v || !aligned(x, v) || !aligned(rows, v))) v /= 2;
  c.ld_x = ld_x / v, c.ld_rows = ld_rows / v, c.units = (int)(row / v);
  cudaError_t err;
  if (v == 16) err = run_dispatch<uint4>(s, c, r->n_layers, h.cta, st);
  else if (v == 8) err = run_dispatch<uint2>(s, c, r->n_layers, h.cta, st);
  else if (v == 4) err = run_dispatch<uint32_t>(s, c, r->n_layers, h.cta, st);
  else if (v == 2) err = run_dispatch<uint16_t>(s, c, r->n_layers, h.cta, st);
  else err = run_dispatch<uint8_t>(s, c, r->n_layers, h.cta, st);
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
