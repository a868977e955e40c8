// Token rows sorted by expert, the rows brought back to their tokens with weights (Eq. 1's sum), and its gradient.
#include <type_traits>

#include "common.cuh"
#include "vec.cuh"

namespace mcce {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMaxRowD = 1 << 24;

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
// One warp per token, or 2, 4 or 8 that share its columns: a warp takes blocks of 32 * V units, every wpt-th block, so that the V
// loads of a lane lie at fixed distances and only the last block of a row needs a look at its end.
struct Token {
  int64_t t, first;   // token over all layers; first sorted row of its layer
  int lane, part;     // this warp's part of the token
  bool there;
  __device__ __forceinline__ Token(int wpt, int64_t tokens, int T, int P) {
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    lane = threadIdx.x & 31;
    t = w / wpt;
    part = (int)w & (wpt - 1);
    there = t < tokens;
    first = there ? t / T * P : 0;
  }
};

struct CopyArgs {
  int64_t ld_x, ld_rows; // in units
  int K, units, scale_cols;
  const void* x;
  void* rows;
  const float* scales;
  float* row_scales;
};

// A row of units narrower than 16 bytes to the positions of its token's pairs, by `parts` warps of which this is number `part`:
// V units of the row are read, all in flight, and written once for every pair, so a token's row is read once.  Full blocks'
// loads and stores lie at fixed distances and need no look at the row's end (8192 x 8 of 1411 bf16: 56 us against
// 73).  What bounds it is the units: 0.57 of the copy bandwidth there with 2 bytes per load and store, 0.78 with 4 (1411 fp32, 81 us), 0.32 with one
// (1411 e4m3, 50 us).
// position_of(k): of pair k, -1: none.
template <typename V_, typename F>
__device__ __forceinline__ void move_row(const CopyArgs& a, int64_t t, int64_t first, int lane, int part, int parts, F position_of) {
  constexpr int V = 8;
  const V_* x = (const V_*)a.x + t * a.ld_x;
  V_* rows = (V_*)a.rows + first * a.ld_rows;
  for (int b = part * 32 * V; b < a.units; b += parts * 32 * V) {
    V_ p[V];
    if (b + 32 * V <= a.units) {
#pragma unroll
      for (int v = 0; v < V; ++v) p[v] = __ldg(x + b + lane + v * 32);
      for (int k = 0; k < a.K; ++k) {
        const int pos = position_of(k);
        if (pos < 0) continue;
        V_* to = rows + pos * a.ld_rows + b + lane;
#pragma unroll
        for (int v = 0; v < V; ++v) to[v * 32] = p[v];
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (b + lane + v * 32 < a.units) p[v] = __ldg(x + b + lane + v * 32);
      for (int k = 0; k < a.K; ++k) {
        const int pos = position_of(k);
        if (pos < 0) continue;
        V_* to = rows + pos * a.ld_rows + b + lane;
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (b + lane + v * 32 < a.units) to[v * 32] = p[v];
      }
    }
  }
}

// Rows of 16-byte units go through shared memory in pieces of kPiece units: fetched by cp.async, which needs no registers and so
// starts before the counting, and written by one bulk copy per pair, issued by as many lanes at once.  Against loads into registers
// and stores of 16 bytes per lane, us: 16384 x 8, a tenth of the pairs dropped, rows of 2048 bytes with scales 54.8 / 58, of 4096 bytes 94.3 / 99; 24 x 256
// tokens x 4 of 4096 bytes 24.4 / 24.8; 20000 x 8 of 1024 bytes to 256 experts 48.1 / 46.7 (half of a piece's lanes idle).  Pieces of 64 units, three
// per warp: 56.2, 95.0, 24.2 and 46.1.
constexpr int kPiece = 128, kRing = 2;
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void fetch_unit(uint4* to, const uint4* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared_address(to)), "l"(__cvta_generic_to_global(from)) : "memory");
}
__device__ __forceinline__ void bulk_store(void* to, const uint4* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(__cvta_generic_to_global(to)),
               "r"(shared_address(from)), "r"(bytes)
               : "memory");
}

// The pieces that a warp moves, one after the other: number `part` of `parts` warps that share a token.
struct Pieces {
  int t, b;
  __device__ __forceinline__ Pieces(int warp, int part, int parts, int blocks, int n_tok) : t(part < blocks ? warp / parts : n_tok), b(part) {}
  __device__ __forceinline__ void next(int part, int parts, int blocks) {
    b += parts;
    if (b >= blocks) b = part, t += 8 / parts;
  }
};

// Ranks the pairs of a few tokens and moves their rows.  Where a pair goes: pairs of smaller experts (totals of all chunks), of
// its expert in earlier chunks (both from the chunks' counts), earlier in its chunk (counted here again), earlier in this
// CTA.  A layer of few pairs is one chunk: the CTA counts all of it, and there is no launch before this one.
// A pair's rank among its CTA's pairs comes from its warp's matches and the counts of the warps before.
// Bound: HBM writes, once the counting is done: 16384 x 8, a tenth dropped, rows of 4096 bytes 94.3 us (0.89 of the copy bandwidth), of
// 2048 bytes with scales 55 (0.79); about 8 us of each are the counting launch and the wait for the first CTAs' positions.  More CTAs per SM
// at once are slower, not faster: 5 / 6 / 8 of them 99 / 101 / 115 with 4096 bytes (before the bulk copies).
constexpr int kCtaPairs = 128;    // pairs of a CTA at most
template <typename V>
__global__ void __launch_bounds__(256) rows_dispatch_kernel(const __grid_constant__ SortArgs s, const __grid_constant__ CopyArgs a,
                                                            const int tokens_per_cta) {
  __shared__ int total[kMaxE], before[kMaxE], warp_sum[8], place[kCtaPairs], in_warp[4][kMaxE];
  const int l = blockIdx.y, t0 = blockIdx.x * tokens_per_cta, n_tok = min(tokens_per_cta, s.T - t0);
  const int q0 = t0 * s.K, n = n_tok * s.K, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = t0 / s.chunk, chunk0 = b * s.chunk * s.K;
  const int32_t* sel = s.sel + (size_t)l * s.P;
  const int64_t first = (int64_t)l * s.P;
  // one warp per token for eight tokens or more, else the eight warps shared out
  const int parts = n_tok >= 8 ? 1 : n_tok >= 4 ? 2 : n_tok >= 2 ? 4 : 8, part = warp & (parts - 1);
  constexpr bool kBulk = sizeof(V) == 16;
  __shared__ uint4 ring[kBulk ? 8 * kRing * kPiece : 1];
  uint4* mine = ring + (kBulk ? warp * kRing * kPiece : 0);
  const int blocks = (a.units + kPiece - 1) / kPiece;
  Pieces ahead(warp, part, parts, blocks, n_tok);
  auto fetch = [&](int slot) {
    if (ahead.t < n_tok) {
      const uint4* x = (const uint4*)a.x + ((int64_t)l * s.T + t0 + ahead.t) * a.ld_x;
#pragma unroll
      for (int v = 0; v < kPiece / 32; ++v) {
        const int u = lane + 32 * v;
        if (ahead.b * kPiece + u < a.units) fetch_unit(mine + slot * kPiece + u, x + ahead.b * kPiece + u);
      }
      ahead.next(part, parts, blocks);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int e_mine = -1, rank = 0;
  if (tid < n) e_mine = sel[q0 + tid];
  if ((unsigned)e_mine >= (unsigned)s.E) e_mine = -1;
  if constexpr (kBulk) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) fetch(i);
  }
  total[tid] = before[tid] = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) in_warp[w][tid] = 0;
  __syncthreads();
  if (warp * 32 < n) {
    const unsigned same = __match_any_sync(kFull, e_mine);
    rank = __popc(same & ((1u << lane) - 1));
    if (e_mine >= 0 && rank == 0) in_warp[warp][e_mine] = __popc(same);
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
    int pos = -1;
    if (e_mine >= 0) {
      pos = before[e_mine] + rank;
      for (int w = 0; w < warp; ++w) pos += in_warp[w][e_mine];
    }
    place[tid] = pos;
    s.inv[(size_t)l * s.P + q0 + tid] = pos;
    if (s.perm && pos >= 0) s.perm[(size_t)l * s.P + pos] = q0 + tid;
  }
  __syncthreads();
  if constexpr (kBulk) {
    int slot = 0;
    for (Pieces p(warp, part, parts, blocks, n_tok); p.t < n_tok; p.next(part, parts, blocks)) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      const int pos = lane < s.K ? place[p.t * s.K + lane] : -1;
      if (pos >= 0)
        bulk_store((uint4*)a.rows + (first + pos) * a.ld_rows + p.b * kPiece, mine + slot * kPiece, min(kPiece, a.units - p.b * kPiece) * 16);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      if (ahead.t < n_tok) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
      }
      fetch(slot);
      slot = slot + 1 == kRing ? 0 : slot + 1;
    }
  } else if (a.x) {
    for (int t = warp / parts; t < n_tok; t += 8 / parts)
      move_row<V>(a, (int64_t)l * s.T + t0 + t, first, lane, part, parts, [&](int k) { return place[t * s.K + k]; });
  }
  if (a.scale_cols) {
    const int k0 = (part * 32 + lane) / a.scale_cols, i0 = (part * 32 + lane) % a.scale_cols;
    const int dk = parts * 32 / a.scale_cols, di = parts * 32 % a.scale_cols;
    for (int t = warp / parts; t < n_tok; t += 8 / parts) {
      const float* from = a.scales + ((int64_t)l * s.T + t0 + t) * a.scale_cols;
      int i = i0;
#pragma unroll 4
      for (int k = k0; k < s.K; k += dk) {
        const int pos = place[t * s.K + k];
        if (pos >= 0) a.row_scales[(first + pos) * a.scale_cols + i] = __ldg(from + i);
        i += di;
        if (i >= a.scale_cols) i -= a.scale_cols, ++k;
      }
    }
  }
  if constexpr (kBulk) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

struct CombineArgs {
  int64_t tokens, ld_token, ld_rows;
  int T, K, P, d, wpt;
  const int32_t* inv;
  const float* w;
  const void *rows, *add;
  void* y;
  const void* dy;
  void* drows;
  float* dw;
};

// The pairs of a token in the lanes of its warp: position (-1: none) and weight.
struct Pairs {
  int pos;
  float w;
  __device__ __forceinline__ Pairs(const CombineArgs& a, const Token& tk) : pos(-1), w(1.f) {
    if (tk.there && tk.lane < a.K) {
      const int p = a.inv[tk.t * a.K + tk.lane];
      if ((unsigned)p < (unsigned)a.P) {
        pos = p;
        if (a.w) w = a.w[tk.t * a.K + tk.lane];
      }
    }
  }
  // of pair k, the same in all lanes
  __device__ __forceinline__ int position(int k, int K) const {
    const int p = __shfl_sync(kFull, pos, k & 31);
    return k < K ? p : -1;
  }
  __device__ __forceinline__ float weight(int k) const { return __shfl_sync(kFull, w, k & 31); }
};

template <int U>
__device__ __forceinline__ void add_scaled(float2 (&s)[(U + 1) / 2], const float2 (&e)[(U + 1) / 2], float w) {
  if constexpr (U == 1) {
    s[0].x = fmaf(e[0].x, w, s[0].x);
  } else {
#pragma unroll
    for (int j = 0; j < U / 2; ++j) s[j] = fma2(e[j], both(w), s[j]);
  }
}

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(__cvta_generic_to_global(p))); }

// y of a token: U columns (16 bytes of a row) at a time, VPT such units per lane and KC rows at once, so that KC * VPT loads are in flight.
template <typename T, typename Y, int U, int KC, int VPT>
__global__ void __launch_bounds__(256) combine_rows_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int N = U / 2;
  const Token tk(a.wpt, a.tokens, a.T, a.P);
  const Pairs pairs(a, tk);
  const T* rows = (const T*)a.rows + tk.first * a.ld_rows;
  const int64_t at = tk.t * a.ld_token;
  const int d = tk.there ? a.d : 0, step = a.wpt * 32 * U;
  for (int b = 0; b < a.d; b += step * VPT) {
    const int c0 = b + (tk.part * 32 + tk.lane) * U;
    float2 s[VPT][N];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int j = 0; j < N; ++j) s[v][j] = both(0.f);
    // The sum's last term is loaded last (held meanwhile, it costs a CTA per SM), but asked for into L2 at once.  K = 6 with a tenth of
    // the pairs dropped, us: not asked for 89.7, asked for 86.0, loaded here 95.3; K = 8, none dropped: 108.4, 105.3, 119.1.  One row at a time: worse (K = 2 28.8, 36.5).
    if constexpr (KC > 1) {
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        if (a.add && c0 + v * step < d) prefetch_l2((const Y*)a.add + at + c0 + v * step);
    }
    for (int k0 = 0; k0 < a.K; k0 += KC) {
      Pack<T, U> p[KC][VPT];
      float w[KC];
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const int pos = k0 + k < a.K ? __shfl_sync(kFull, pairs.pos, k0 + k) : -1;
        w[k] = __shfl_sync(kFull, pairs.w, (k0 + k) & 15);
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

// The same for narrower units (odd widths, unaligned rows), where instructions are what bounds it: blocks that lie inside the row and
// whose pairs all have rows run without a predicate, at fixed distances.
template <typename T, typename Y, int U, int KC, int VPT>
__global__ void __launch_bounds__(256) combine_narrow_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int N = (U + 1) / 2, kBlock = 32 * U * VPT;
  const Token tk(a.wpt, a.tokens, a.T, a.P);
  const Pairs pairs(a, tk);
  const T* rows = (const T*)a.rows + tk.first * a.ld_rows + tk.lane * U;
  const int64_t at = tk.t * a.ld_token + tk.lane * U;
  const int d = tk.there ? a.d : 0;
  auto block = [&](int b, auto whole) {   // columns b .. b + kBlock, all of them inside the row or not
    constexpr bool kWhole = decltype(whole)::value;
    const int left = d - b - tk.lane * U;
    float2 s[VPT][N];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int j = 0; j < N; ++j) s[v][j] = both(0.f);
    for (int k0 = 0; k0 < a.K; k0 += KC) {
      int pos[KC], least = 0;
      float w[KC];
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        pos[k] = pairs.position(k0 + k, a.K);
        w[k] = pairs.weight(k0 + k);
        least = min(least, pos[k]);
      }
      // (branches between the loads would keep them from being issued together: either none, or predicates)
      auto rows_of = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        Pack<T, U> p[KC][VPT];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const T* row = rows + pos[k] * a.ld_rows + b;
#pragma unroll
          for (int v = 0; v < VPT; ++v) {
            if (!kAll) p[k][v].zero();
            if (kAll || (pos[k] >= 0 && v * 32 * U < left)) p[k][v].load_const(row + v * 32 * U);
          }
        }
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
          for (int v = 0; v < VPT; ++v) {
            float2 e[N];
            p[k][v].get(e);
            add_scaled<U>(s[v], e, w[k]);
          }
      };
      if constexpr (kWhole) {
        if (least == 0) rows_of(std::true_type{});
        else rows_of(std::false_type{});
      } else {
        rows_of(std::false_type{});
      }
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if (!kWhole && v * 32 * U >= left) continue;
      Pack<Y, U> y;
      if (a.add) {
        y.load((const Y*)a.add + at + b + v * 32 * U);
        float2 e[N];
        y.get(e);
#pragma unroll
        for (int j = 0; j < N; ++j) s[v][j] = add2(s[v][j], e[j]);
      }
      y.set(s[v]);
      y.store((Y*)a.y + at + b + v * 32 * U);
    }
  };
  for (int b = tk.part * kBlock; b < a.d; b += a.wpt * kBlock) {
    if (b + kBlock <= d) block(b, std::true_type{});
    else block(b, std::false_type{});
  }
}

// Sums of acc[k] over a warp, k < KC.  The number of values is halved while the lanes that share one double, so KC sums
// cost little more than one; lane l holds that of k = l / (32 / KC) afterwards.
template <int KC>
__device__ __forceinline__ float sum_of_all(float (&acc)[KC]) {
  int o = 16;
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
// Bound: HBM (0.98 of the copy bandwidth on 16384 x 8 rows of 2048 bf16, half of it writes).
template <typename T, typename Y, int U, int KC, int VPT>
__global__ void __launch_bounds__(256) combine_rows_grad_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int N = (U + 1) / 2, kBlock = 32 * U * VPT;
  __shared__ float parts[8][KC];
  const Token tk(a.wpt, a.tokens, a.T, a.P);
  const Pairs pairs(a, tk);
  const Y* dy = (const Y*)a.dy + tk.t * a.ld_token + tk.lane * U;
  const int d = tk.there ? a.d : 0;
  for (int k0 = 0; k0 < a.K; k0 += KC) {
    int64_t at[KC];   // this lane's first element of the pair's row, -1: no row
    float w[KC], acc[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const int pos = pairs.position(k0 + k, a.K);
      w[k] = pairs.weight(k0 + k);
      at[k] = pos >= 0 ? (tk.first + pos) * a.ld_rows + tk.lane * U : -1;
      acc[k] = 0.f;
    }
    bool all_there = true;
#pragma unroll
    for (int k = 0; k < KC; ++k) all_there &= at[k] >= 0;
    auto block = [&](int b, auto all) {   // all: every pair has a row and all columns of the block lie in it
      constexpr bool kAll = decltype(all)::value;
      const int left = d - b - tk.lane * U;
      Pack<T, U> p[KC][VPT];
      Pack<Y, U> q[VPT];
#pragma unroll
      for (int v = 0; v < VPT; ++v)
        if (kAll || v * 32 * U < left) q[v].load_const(dy + b + v * 32 * U);
      if (a.dw) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const T* row = (const T*)a.rows + at[k] + b;
#pragma unroll
          for (int v = 0; v < VPT; ++v)
            if (kAll || (at[k] >= 0 && v * 32 * U < left)) p[k][v].load(row + v * 32 * U);
        }
      }
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        T* row = (T*)a.drows + at[k] + b;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
          if (!kAll && (at[k] < 0 || v * 32 * U >= left)) continue;
          float2 g[N], e[N];
          q[v].get(g);
          if (a.dw) {
            p[k][v].get(e);
            if constexpr (U == 1) {
              acc[k] = fmaf(e[0].x, g[0].x, acc[k]);
            } else {
              float2 s = both(0.f);
#pragma unroll
              for (int j = 0; j < N; ++j) s = fma2(e[j], g[j], s);
              acc[k] += s.x + s.y;
            }
          }
#pragma unroll
          for (int j = 0; j < N; ++j) e[j] = U == 1 ? make_float2(g[j].x * w[k], 0.f) : mul2(g[j], both(w[k]));
          p[k][v].set(e);
          p[k][v].store(row + v * 32 * U);
        }
      }
    };
    for (int b = tk.part * kBlock; b < d; b += a.wpt * kBlock) {
      // (a look at the row's end costs little beside the columns of a 16-byte unit)
      if (U * sizeof(T) < 16 && all_there && b + kBlock <= d) block(b, std::true_type{});
      else block(b, std::false_type{});
    }
    if (!a.dw) continue;
    const float s = sum_of_all(acc);
    const int k = tk.lane / (32 / KC);
    const bool speaks = tk.lane % (32 / KC) == 0 && tk.there && k0 + k < a.K;
    if (a.wpt == 1) {
      if (speaks) a.dw[tk.t * a.K + k0 + k] = s;
    } else {
      __syncthreads();   // the last chunk's parts have been read
      if (speaks) parts[threadIdx.x >> 5][k] = s;
      __syncthreads();
      if (speaks && tk.part == 0) {
        float v = 0.f;
        for (int i = 0; i < a.wpt; ++i) v += parts[(threadIdx.x >> 5) + i][k];
        a.dw[tk.t * a.K + k0 + k] = v;
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
  if (r->n_layers < 1 || r->n_layers > 65535 || r->n_tokens < 0 || r->top_k < 1 || r->top_k > kMaxK || r->d < 1 || r->d > kMaxRowD)
    return false;
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
// A CTA moves up to 150 KB: 16384 tokens x 8, a tenth of the pairs dropped, of 2048 bytes with scales, us, 4 / 8 / 16 tokens: 58.7 / 54.9 / 58.0; of 4096 bytes
// 2 / 4 / 8 tokens: 106 / 94.0 / 95.2; 24 x 256 tokens x 4 of 4096 bytes 2 / 4 tokens 26.1 / 24.3.
// Chunks of 2048 pairs: between 512 and 4096 the time changes by 1 %.  A layer is one chunk -- one launch, every CTA counts
// the whole layer -- while that is little work: 24 x 256 tokens x 4 25.0 against 27.9 with two launches, 4096 tokens x 2 of 8192
// bytes 32.7 against 22.8.
SortShape sort_shape(const mcce_rows& r) {
  const int K = r.top_k, T = r.n_tokens;
  const int64_t moved = (int64_t)(K + 1) * r.d * (r.dtype == MCCE_F32 ? 4 : r.dtype == MCCE_BF16 ? 2 : 1);
  SortShape h;
  h.cta = 1;
  while (h.cta * 2 * K <= kCtaPairs && h.cta * 2 * moved <= 150 * 1024) h.cta *= 2;
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

// Warps per token: a power of two that covers the row's units `per_lane` at a time, at most 8.
int warps_per_token(int units, int per_lane) {
  int w = 1;
  while (w < 8 && w * 32 * per_lane < units) w *= 2;
  return w;
}
template <typename K>
cudaError_t launch_tokens(K kernel, const CombineArgs& a, cudaStream_t st) {
  const int64_t grid = (a.tokens * a.wpt + 7) / 8;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  kernel<<<(unsigned)grid, 256, 0, st>>>(a);
  return cudaGetLastError();
}

// With fewer tokens than this the device is not full: one unit per lane and as many warps per token as that takes.
bool few(const CombineArgs& a) { return a.tokens * 64 < 148 * 1024; }

// KC rows at once x VPT units at once, us measured back to back on rotating buffers (16384 tokens of 2048 bf16 columns unless
// noted).  Return, K = 8: 4 x 1 with 2 warps per token 94.6 (0.98 of the copy bandwidth), 8 x 1 104, 2 x 2 133; K = 6 with add (before it was asked for early): 4 x 1
// 92.4, 3 x 1 92.3, 1 x 2 94.1; K = 2, 4099 tokens of 4096: 1 x 2 22.1 (0.69), 2 x 2 22.7, 4 x 1 24.8; K = 1 of 4096: 1 x 4 49.2 (0.83); 256
// tokens, K = 8: 4 x 1 with 8 warps 4.2, 4 x 2 4.7.  Gradient, K = 8: 1 x 4 with 2 warps 177 (0.98), 2 x 2 181, 4 x 1 191; K = 1 of 4096: 1 x 4
// 63.6 (0.97); 256 tokens, K = 8: 4 x 1 with 8 warps 6.3, 2 x 2 8.3.
// Units of one bf16: 8192 tokens of 1411, K = 8, return 4 x 8 with 2 warps 51.4 (0.62), 4 x 4 57, 1 x 8 62; of 4097, K = 2: 2 x 8 49.2 (0.62), 1 x 8 53;
// gradient 4 x 4 106 (0.57), 2 x 4 117; K = 2: 2 x 4 86 (0.59).  Sixteen-byte loads at the next boundary, shifted into place: 74 and 166.
// A width that 4 divides but not 8 has units of two bf16: 16384 x 8 of 1004 55 (0.82) and 123 (0.70), of 1000 52 and 97.
template <typename T, typename Y, int U>
cudaError_t run_combine(CombineArgs a, cudaStream_t st) {
  const int units = (a.d + U - 1) / U;
  if constexpr (U * sizeof(T) == 16) {
    a.wpt = warps_per_token(units, few(a) ? 1 : 4);
    if (a.K == 1) return launch_tokens(combine_rows_kernel<T, Y, U, 1, 4>, a, st);
    if (a.K == 2) return launch_tokens(combine_rows_kernel<T, Y, U, 1, 2>, a, st);
    return launch_tokens(combine_rows_kernel<T, Y, U, 4, sizeof(T) == 4 ? 2 : 1>, a, st);
  } else {
    a.wpt = warps_per_token(units, few(a) ? 1 : 36);
    if (a.K <= 2) return launch_tokens(combine_narrow_kernel<T, Y, U, 2, 8 / U>, a, st);
    return launch_tokens(combine_narrow_kernel<T, Y, U, 4, sizeof(T) == 4 ? 4 : 8 / U>, a, st);
  }
}
template <typename T, typename Y, int U>
cudaError_t run_combine_grad(CombineArgs a, cudaStream_t st) {
  const int units = (a.d + U - 1) / U;
  if constexpr (U * sizeof(T) == 16) {
    if (few(a)) return a.wpt = warps_per_token(units, 1), launch_tokens(combine_rows_grad_kernel<T, Y, U, 4, 1>, a, st);
    a.wpt = units > 128 ? 2 : 1;
    return launch_tokens(combine_rows_grad_kernel<T, Y, U, 1, 4>, a, st);
  } else {
    a.wpt = warps_per_token(units, few(a) ? 1 : 36);
    if (a.K <= 2) return launch_tokens(combine_rows_grad_kernel<T, Y, U, 2, 4>, a, st);
    return launch_tokens(combine_rows_grad_kernel<T, Y, U, 4, 4 / U>, a, st);
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

// A launch that follows the kernel before it at once: it starts when that one's last CTAs end, without the time between two launches, and waits
// for its memory itself.  (No kernel here lets its dependents start sooner.)
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
  const int64_t tokens = (int64_t)r->n_layers * r->n_tokens, pairs = tokens * r->top_k;
  const Span ssel = flat_span(sel_idx, pairs * 4), sx = row_span(x, tokens, ld_or(r->ld_token, r->d), r->d, e);
  const Span ssc = flat_span(scales, tokens, 4ll * r->scale_cols), soff = flat_span(offsets, (int64_t)r->n_layers * (r->n_experts + 1) * 4);
  const Span sperm = flat_span(perm, pairs * 4), sinv = flat_span(inv, pairs * 4);
  const Span srows = row_span(rows, pairs, ld_or(r->ld_rows, r->d), r->d, e), sosc = flat_span(row_scales, pairs, 4ll * r->scale_cols);
  const Span sws = flat_span(need ? workspace : nullptr, need);
  if (!apart(soff, {&ssel, &sx, &ssc, &sperm, &sinv, &srows, &sosc}) || !apart(sperm, {&ssel, &sx, &ssc, &sinv, &srows, &sosc}) ||
      !apart(sinv, {&ssel, &sx, &ssc, &srows, &sosc}) || !apart(srows, {&ssel, &sx, &ssc, &sosc}) || !apart(sosc, {&ssel, &sx, &ssc}) ||
      !apart(sws, {&ssel, &sx, &ssc, &soff, &sperm, &sinv, &srows, &sosc}))
    return MCCE_EINVAL;
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
  const int64_t pairs = a.tokens * a.K;
  const Span sy = row_span(y, a.tokens, a.ld_token, a.d, ey), sadd = row_span(add, a.tokens, a.ld_token, a.d, ey);
  const Span srows = row_span(rows, pairs, a.ld_rows, a.d, e), sinv = flat_span(inv, pairs * 4), sw = flat_span(sel_w, pairs * 4);
  if (!same_or_apart(sy, sadd) || !apart(sy, {&srows, &sinv, &sw})) return MCCE_EINVAL;
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
  const int64_t pairs = a.tokens * a.K;
  const Span sdy = row_span(dy, a.tokens, a.ld_token, a.d, ey), srows = row_span(dw ? rows : nullptr, pairs, a.ld_rows, a.d, e);
  const Span sinv = flat_span(inv, pairs * 4), sw = flat_span(sel_w, pairs * 4), sdr = row_span(drows, pairs, a.ld_rows, a.d, e);
  const Span sdw = flat_span(dw, pairs * 4);
  if (!same_or_apart(sdr, srows) || !apart(sdr, {&sdy, &sinv, &sw}) || !apart(sdw, {&sdy, &srows, &sinv, &sw, &sdr}))
    return MCCE_EINVAL;
  a.inv = inv, a.w = sel_w, a.rows = dw ? rows : nullptr, a.dy = dy, a.drows = drows, a.dw = dw;
  UnitRule u(r->d, 16 / e);
  u.tensor(a.rows, a.ld_rows, e);
  u.tensor(drows, a.ld_rows, e);
  u.tensor(dy, a.ld_token, ey);
  return run_combine_types(*r, a, u.u, true, (cudaStream_t)cuda_stream) == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
