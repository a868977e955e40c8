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
// elements of a row that starts at element `at` of a tensor before its first whole unit
template <int U>
__device__ __forceinline__ int head_of(int64_t at, int off, int d) { return min(d, (int)(-(at + off) & (U - 1))); }

struct CopyArgs {
  int64_t tokens;        // L * T
  int64_t ld_x, ld_rows;
  int T, K, P, d, scale_cols, tpt, off;   // off: of rows, in elements, past a 16-byte boundary
  const int32_t* inv;
  const void* x;
  void* rows;
  const float* scales;
  float* row_scales;
};

__device__ __forceinline__ void copy_scales(const CopyArgs& a, const Token& tk, int k, int pos) {
  for (int c = tk.u0; c < a.scale_cols; c += a.tpt)
    a.row_scales[(tk.first + pos) * a.scale_cols + c] = a.scales[tk.t * a.scale_cols + c];
}

// A token's row is read once, a unit of 16 bytes per thread, and written to the positions of its pairs.  RAGGED: the
// units are those of the destination, whose alignment differs from pair to pair, shifted out of the token's row.
template <typename T, bool RAGGED>
__global__ void __launch_bounds__(256) rows_copy_kernel(const __grid_constant__ CopyArgs a) {
  constexpr int U = 16 / (int)sizeof(T);
  cudaGridDependencySynchronize();
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  const T* x = (const T*)a.x + tk.t * a.ld_x;
  T* rows = (T*)a.rows + tk.first * a.ld_rows;
  if (!RAGGED && a.x) {
    const int n = tk.there ? a.d / U : 0, rounds = (a.d / U + a.tpt - 1) / a.tpt;
    for (int i = 0, u = tk.u0; i < rounds; ++i, u += a.tpt) {
      Pack<T, U> v;
      if (u < n) v.load_const(x + u * U);
      for (int k = 0; k < a.K; ++k) {
        const int pos = position(tk, mine, k);
        if (pos >= 0 && u < n) v.store(rows + pos * a.ld_rows + u * U);
      }
    }
  }
  for (int k = 0; k < a.K; ++k) {
    const int pos = position(tk, mine, k);
    if (pos < 0) continue;
    if (RAGGED && a.x) {
      const int head = head_of<U>((tk.first + pos) * a.ld_rows, a.off, a.d), whole = (a.d - head) & ~(U - 1);
      T* row = rows + pos * a.ld_rows;
      const T* end = (const T*)a.x + (a.tokens - 1) * a.ld_x + a.d;
      for (int c = head + tk.u0 * U; c < head + whole; c += a.tpt * U) {
        Pack<T, U> v;
        load_anywhere(v, x + c, (const T*)a.x, end);
        v.store(row + c);
      }
      if (tk.u0 < head) row[tk.u0] = x[tk.u0];
      if (head + whole + tk.u0 < a.d) row[head + whole + tk.u0] = x[head + whole + tk.u0];
    }
    copy_scales(a, tk, k, pos);
  }
}

// Few pairs per layer: one launch.  Every CTA counts all pairs of its layer (and, in the upper half of a word, those before
// its own tokens), ranks its own and moves their rows; the counting takes the place of two more launches.
constexpr int kFusedPairs = 64;    // pairs of a CTA at most
template <typename T, bool RAGGED>
__global__ void __launch_bounds__(256) rows_dispatch_kernel(const __grid_constant__ SortArgs s, const __grid_constant__ CopyArgs a,
                                                            const int tokens_per_cta) {
  constexpr int U = 16 / (int)sizeof(T);
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
  const int64_t first = (int64_t)l * s.P;
  const T* end = (const T*)a.x + (a.tokens - 1) * a.ld_x + a.d;
  if (a.x) {
    if (!RAGGED) {
      const int units = a.d / U;
      for (int i = tid; i < n_tok * units; i += 256) {
        const int t = i / units, u = i - t * units;
        Pack<T, U> v;
        v.load_const((const T*)a.x + ((int64_t)l * s.T + t0 + t) * a.ld_x + u * U);
        for (int k = 0; k < s.K; ++k) {
          const int pos = place[t * s.K + k];
          if (pos >= 0) v.store((T*)a.rows + (first + pos) * a.ld_rows + u * U);
        }
      }
    } else {
      for (int p = warp; p < n; p += 8) {   // a warp per pair
        const int pos = place[p];
        if (pos < 0) continue;
        const T* x = (const T*)a.x + ((int64_t)l * s.T + t0 + p / s.K) * a.ld_x;
        T* row = (T*)a.rows + (first + pos) * a.ld_rows;
        const int head = head_of<U>((first + pos) * a.ld_rows, a.off, a.d), whole = (a.d - head) & ~(U - 1);
        for (int col = head + lane * U; col < head + whole; col += 32 * U) {
          Pack<T, U> v;
          load_anywhere(v, x + col, (const T*)a.x, end);
          v.store(row + col);
        }
        if (lane < head) row[lane] = x[lane];
        if (head + whole + lane < a.d) row[head + whole + lane] = x[head + whole + lane];
      }
    }
  }
  for (int i = tid; i < n * a.scale_cols; i += 256) {
    const int p = i / a.scale_cols, col = i - p * a.scale_cols, pos = place[p];
    if (pos >= 0)
      a.row_scales[(first + pos) * a.scale_cols + col] = a.scales[((int64_t)l * s.T + t0 + p / s.K) * a.scale_cols + col];
  }
}

struct CombineArgs {
  int64_t tokens, ld_token, ld_rows;
  int T, K, P, d, tpt, off;   // off: of y or of drows, in elements, past a unit's boundary
  const int32_t* inv;
  const float* w;
  const void *rows, *add;
  void* y;
  const void* dy;
  void* drows;
  float* dw;
};

// y of a token: VPT units per thread and KC rows at a time, so that about eight 16-byte loads are in flight per thread.
// RAGGED: the units are those of y; the rows, whose alignment differs from pair to pair, are shifted into place.
template <typename T, typename Y, int KC, int VPT, bool RAGGED>
__global__ void __launch_bounds__(256) combine_rows_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int U = 16 / (int)sizeof(T);
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  const int pair = (int)(threadIdx.x & 31) - tk.lane0;
  const float my_w = mine >= 0 && a.w ? a.w[tk.t * a.K + pair] : 1.f;
  const T* rows = (const T*)a.rows + tk.first * a.ld_rows;
  const T* end = (const T*)a.rows + (a.tokens / a.T * a.P - 1) * a.ld_rows + a.d;
  const int64_t at = tk.t * a.ld_token;
  const int d = tk.there ? a.d : 0;
  const int head = RAGGED ? head_of<U>(at, a.off, d) : 0, whole = RAGGED ? (d - head) & ~(U - 1) : d;
  const int per_round = a.tpt * U * VPT, rounds = (a.d + per_round - 1) / per_round;
  for (int i = 0; i < rounds; ++i) {
    const int c0 = i * per_round + tk.u0 * U;
    float2 s[VPT][U / 2];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int j = 0; j < U / 2; ++j) s[v][j] = both(0.f);
    for (int k0 = 0; k0 < a.K; k0 += KC) {
      Pack<T, U> p[KC][VPT];
      float w[KC];
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const int pos = k0 + k < a.K ? position(tk, mine, k0 + k) : -1;
        w[k] = __shfl_sync(kFull, my_w, tk.lane0 + ((k0 + k) & 15));
        const T* row = rows + pos * a.ld_rows + head + c0;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          p[k][v].zero();
          if (pos >= 0 && c0 + v * a.tpt * U < whole) {
            if constexpr (RAGGED) load_anywhere(p[k][v], row + v * a.tpt * U, (const T*)a.rows, end);
            else p[k][v].load_const(row + v * a.tpt * U);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          float2 e[U / 2];
          p[k][v].get(e);
#pragma unroll
          for (int j = 0; j < U / 2; ++j) s[v][j] = fma2(e[j], both(w[k]), s[v][j]);
        }
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = c0 + v * a.tpt * U;
      if (c >= whole) continue;
      Pack<Y, U> y;
      if (a.add) {
        const Y* add = (const Y*)a.add + at + head + c;
        if constexpr (RAGGED) load_anywhere(y, add, (const Y*)a.add, (const Y*)a.add + (a.tokens - 1) * a.ld_token + a.d);
        else y.load(add);
        float2 e[U / 2];
        y.get(e);
#pragma unroll
        for (int j = 0; j < U / 2; ++j) s[v][j] = add2(s[v][j], e[j]);
      }
      y.set(s[v]);
      y.store((Y*)a.y + at + head + c);
    }
  }
  if (RAGGED) {   // single elements of the row's first U threads
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int c = side ? head + whole + tk.u0 : tk.u0;
      const bool in = side ? c < d : tk.u0 < head;
      float s = 0.f;
      for (int k = 0; k < a.K; ++k) {
        const int pos = position(tk, mine, k);
        const float w = __shfl_sync(kFull, my_w, tk.lane0 + k);
        if (in && pos >= 0) s = fmaf(wide(rows[pos * a.ld_rows + c]), w, s);
      }
      if (in) ((Y*)a.y)[at + c] = narrow<Y>(a.add ? s + wide(((const Y*)a.add)[at + c]) : s);
    }
  }
}

// Sum of acc[k] over the lanes of a token, k < KC; lane l of a group of KC holds that of k = bit-reversed l afterwards.
template <int KC>
__device__ __forceinline__ float sum_of_all(float (&acc)[KC], int lanes) {
  // halve the number of values and double the lanes that share one, until one is left
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

// drows and dw of a token: a row's unit is read, multiplied into the pair's sum, and replaced by w dy.  KC rows at a time.
// RAGGED: the units are those of the sorted rows; dy, which lies in L1 after the first pair, is shifted into place.
template <typename T, typename Y, int KC, bool RAGGED>
__global__ void __launch_bounds__(256) combine_rows_grad_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int U = 16 / (int)sizeof(T);
  __shared__ float parts[8][KC];
  const Token tk(a.tpt, a.tokens, a.T, a.P);
  const int lane = threadIdx.x & 31, lanes = min(a.tpt, 32);
  const int mine = my_position(tk, a.inv, a.K, a.P);
  const float my_w = mine >= 0 && a.w ? a.w[tk.t * a.K + lane - tk.lane0] : 1.f;
  const T* rows = (const T*)a.rows;
  const T* rows_end = rows + (a.tokens / a.T * a.P - 1) * a.ld_rows + a.d;
  T* drows = (T*)a.drows;
  const Y* dy = (const Y*)a.dy + tk.t * a.ld_token;
  const Y* dy_end = (const Y*)a.dy + (a.tokens - 1) * a.ld_token + a.d;
  for (int k0 = 0; k0 < a.K; k0 += KC) {
    int64_t at[KC];   // first element of the pair's row, -1: no row
    int head[KC], whole[KC];
    float w[KC], acc[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const int pos = k0 + k < a.K ? position(tk, mine, k0 + k) : -1;
      w[k] = __shfl_sync(kFull, my_w, tk.lane0 + ((k0 + k) & 15));
      at[k] = pos >= 0 ? (tk.first + pos) * a.ld_rows : -1;
      head[k] = RAGGED && pos >= 0 ? head_of<U>(at[k], a.off, a.d) : 0;
      whole[k] = pos < 0 ? 0 : RAGGED ? (a.d - head[k]) & ~(U - 1) : a.d;
      acc[k] = 0.f;
    }
    for (int c = tk.u0 * U; c < a.d; c += a.tpt * U) {
      Pack<T, U> p[KC];
      float2 g[U / 2];
      if (!RAGGED && tk.there) {
        Pack<Y, U> q;
        q.load_const(dy + c);
        q.get(g);
      }
      if (a.dw) {
#pragma unroll
        for (int k = 0; k < KC; ++k)
          if (c < whole[k]) {
            if constexpr (RAGGED) load_anywhere(p[k], rows + at[k] + head[k] + c, rows, rows_end);
            else p[k].load(rows + at[k] + c);
          }
      }
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        if (c >= whole[k]) continue;
        if constexpr (RAGGED) {
          Pack<Y, U> q;
          load_anywhere(q, dy + head[k] + c, (const Y*)a.dy, dy_end);
          q.get(g);
        }
        float2 e[U / 2];
        if (a.dw) {
          p[k].get(e);
          float2 s = both(0.f);
#pragma unroll
          for (int j = 0; j < U / 2; ++j) s = fma2(e[j], g[j], s);
          acc[k] += s.x + s.y;
        }
#pragma unroll
        for (int j = 0; j < U / 2; ++j) e[j] = mul2(g[j], both(w[k]));
        p[k].set(e);
        p[k].store(drows + at[k] + head[k] + c);
      }
    }
    if (RAGGED) {
#pragma unroll
      for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          const int c = side ? head[k] + whole[k] + tk.u0 : tk.u0;
          if (at[k] < 0 || !(side ? c < a.d : tk.u0 < head[k])) continue;
          const float g = wide(dy[c]);
          if (a.dw) acc[k] = fmaf(wide(rows[at[k] + c]), g, acc[k]);
          drows[at[k] + c] = narrow<T>(g * w[k]);
        }
    }
    if (!a.dw) continue;
    const float s = sum_of_all(acc, lanes);
    // this lane's pair of the chunk: the halves were taken from the top bit down
    const int k = (lane & (lanes - 1)) / (lanes / KC);
    const bool speaks = (lane & (lanes / KC - 1)) == 0;
    if (a.tpt <= 32) {
      if (speaks && tk.there && k0 + k < a.K) a.dw[tk.t * a.K + k0 + k] = s;
    } else {
      __syncthreads();
      if (speaks) parts[threadIdx.x >> 5][k] = s;
      __syncthreads();
      if (tk.there && tk.u0 < KC && k0 + tk.u0 < a.K) {
        const int warps = a.tpt >> 5, w0 = (threadIdx.x >> 5);
        float v = 0.f;
        for (int i = 0; i < warps; ++i) v += parts[w0 + i][tk.u0];
        a.dw[tk.t * a.K + k0 + tk.u0] = v;
      }
    }
  }
}

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
template <typename K, typename A>
cudaError_t launch_tokens(K kernel, const A& a, cudaStream_t st) {
  const int64_t grid = (a.tokens * a.tpt + 255) / 256;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  kernel<<<(unsigned)grid, 256, 0, st>>>(a);
  return cudaGetLastError();
}

template <typename T, typename Y, bool RAGGED>
cudaError_t run_combine_k(CombineArgs a, cudaStream_t st) {
  const int units = (a.d * (int)sizeof(T) + 15) / 16;
  if (a.K <= 1) return a.tpt = threads_per_token(units, 4), launch_tokens(combine_rows_kernel<T, Y, 1, 4, RAGGED>, a, st);
  if (a.K <= 2) return a.tpt = threads_per_token(units, 4), launch_tokens(combine_rows_kernel<T, Y, 2, 4, RAGGED>, a, st);
  if (a.K <= 4) return a.tpt = threads_per_token(units, 2), launch_tokens(combine_rows_kernel<T, Y, 4, 2, RAGGED>, a, st);
  return a.tpt = threads_per_token(units, 1), launch_tokens(combine_rows_kernel<T, Y, 8, 1, RAGGED>, a, st);
}
template <typename T, typename Y, bool RAGGED>
cudaError_t run_combine_grad_k(CombineArgs a, cudaStream_t st) {
  const int units = (a.d * (int)sizeof(T) + 15) / 16;
  a.tpt = threads_per_token(units, 4);
  if (a.K <= 1) return launch_tokens(combine_rows_grad_kernel<T, Y, 1, RAGGED>, a, st);
  if (a.K <= 2) return launch_tokens(combine_rows_grad_kernel<T, Y, 2, RAGGED>, a, st);
  if (a.K <= 4) return launch_tokens(combine_rows_grad_kernel<T, Y, 4, RAGGED>, a, st);
  return launch_tokens(combine_rows_grad_kernel<T, Y, 8, RAGGED>, a, st);
}
template <typename T, typename Y>
cudaError_t run_combine(const CombineArgs& a, bool ragged, bool grad, cudaStream_t st) {
  if (grad) return ragged ? run_combine_grad_k<T, Y, true>(a, st) : run_combine_grad_k<T, Y, false>(a, st);
  return ragged ? run_combine_k<T, Y, true>(a, st) : run_combine_k<T, Y, false>(a, st);
}
cudaError_t run_combine_types(const mcce_rows& r, const CombineArgs& a, bool ragged, bool grad, cudaStream_t st) {
  if (r.dtype == MCCE_F32) return run_combine<float, float>(a, ragged, grad, st);
  if (r.token_dtype == MCCE_F32) return run_combine<__nv_bfloat16, float>(a, ragged, grad, st);
  return run_combine<__nv_bfloat16, __nv_bfloat16>(a, ragged, grad, st);
}

// A launch that may begin while the kernel before it ends; the kernel waits for that one itself.
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t st, A... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.stream = st, cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Tokens per CTA of the single launch, 0: several launches.
int fused_tokens(const SortArgs& s, int L) {
  if (s.P > 4096) return 0;
  int t = kFusedPairs / s.K;
  while (t > 1 && (int64_t)((s.T + t - 1) / t) * L < 4 * 148) t = (t + 1) / 2;
  return t;
}

template <typename T>
cudaError_t run_dispatch(const SortArgs& s, CopyArgs c, int L, bool ragged, cudaStream_t st) {
  if (const int t = fused_tokens(s, L)) {
    const dim3 grid((s.T + t - 1) / t, L);
    if (ragged) rows_dispatch_kernel<T, true><<<grid, 256, 0, st>>>(s, c, t);
    else rows_dispatch_kernel<T, false><<<grid, 256, 0, st>>>(s, c, t);
    return cudaGetLastError();
  }
  const dim3 grid(s.B, L);
  rows_count_kernel<<<grid, 256, 0, st>>>(s);
  cudaError_t err = cudaGetLastError();
  if (err == cudaSuccess) err = launch_after(rows_rank_kernel, grid, kSortChunk, st, s);
  if (err != cudaSuccess || !(c.x || c.scale_cols)) return err;
  c.tpt = threads_per_token((c.d * (int)sizeof(T) + 15) / 16, 1);
  const int64_t ctas = (c.tokens * c.tpt + 255) / 256;
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  return ragged ? launch_after(rows_copy_kernel<T, true>, dim3((unsigned)ctas), 256, st, c)
                : launch_after(rows_copy_kernel<T, false>, dim3((unsigned)ctas), 256, st, c);
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
  c.tokens = (int64_t)r->n_layers * r->n_tokens, c.T = s.T, c.K = s.K, c.P = s.P, c.d = r->d, c.scale_cols = r->scale_cols;
  c.ld_x = ld_or(r->ld_token, r->d), c.ld_rows = ld_or(r->ld_rows, r->d);
  c.inv = inv, c.x = x, c.rows = rows, c.scales = scales, c.row_scales = row_scales;
  LayoutRule rule(r->d, 16 / e);
  rule.tensor(rows, c.ld_rows, e);
  c.off = rows ? rule.off : 0;
  rule.tensor(x, c.ld_x, e);
  const bool ragged = x && !rule.aligned;
  cudaError_t err;
  if (e == 4) err = run_dispatch<uint32_t>(s, c, r->n_layers, ragged, st);
  else if (e == 2) err = run_dispatch<uint16_t>(s, c, r->n_layers, ragged, st);
  else err = run_dispatch<uint8_t>(s, c, r->n_layers, ragged, st);
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
  LayoutRule rule(r->d, 16 / e);
  rule.tensor(y, a.ld_token, ey);
  a.off = rule.off;
  rule.tensor(add, a.ld_token, ey);
  rule.tensor(rows, a.ld_rows, e);
  return run_combine_types(*r, a, !rule.aligned, false, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
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
  LayoutRule rule(r->d, 16 / e);
  rule.tensor(drows, a.ld_rows, e);
  a.off = rule.off;
  rule.tensor(a.rows, a.ld_rows, e);
  rule.tensor(dy, a.ld_token, ey);
  return run_combine_types(*r, a, !rule.aligned, true, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
