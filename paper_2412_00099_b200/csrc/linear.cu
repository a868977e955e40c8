// The experts' products on sorted rows: entry points, and the kernels that take any size, stride, alignment and type.
#include "linear.cuh"

#include "span.h"
#include "tc_common.cuh"

namespace mcce {
namespace linear {
namespace {

// ---- products of any shape -----------------------------------------------------------------------------------
// fp32 sums on the fp32 pipe: tiles of 32 x 64, 4 x 4 results per thread, 16 products deep per step.  An operand lies in shared memory as it lies in memory: with
// the reduction along its rows ([row][16], read four products at a time) or across them ([16][row], read four rows at a time); either way 8 16-byte loads
// feed 32 packed multiply-adds.  fp32 operands of the next three steps are on their way by cp.async, 16, 8 or 4 bytes at a time as the alignment allows; bf16
// elements of the next step in registers.  The results go through shared memory so that a warp ends up with 32 neighbouring columns of a row.
// 32 to 42 TFLOP/s (16 groups of 256 rows x 2048 x 512 fp32: 245 us; its gradients 247 and 202), bound by the loads from shared memory and the
// instructions around them; 64 x 64 and 128 x 128 tiles with 8 x 8 results per thread left more SMs idle than they saved (340 and 490 us).
// Where tiles are few, the CTAs of a cluster share a tile's reduction.  900 rows of 10 groups x 1002 x 515 (two elements per copy): 46 to 52 us.
constexpr int kDeep = 16;

template <Kind KIND, typename T, bool GATED>
struct General {
  static constexpr int kSets = KIND == kForward && GATED ? 2 : 1;   // sums per result: a gated forward pass has two
  static constexpr int kThreads = 128, TI = 32, TJ = 64;
  static constexpr int kLanesJ = 16, kLanesI = kThreads / kLanesJ, RI = TI / kLanesI, RJ = TJ / kLanesJ;   // results of a thread
  static constexpr bool kAlongA = KIND != kDweight, kAlongB = KIND == kForward;    // reduction along the operand's rows
  static constexpr int kStrideA = kAlongA ? kDeep + 4 : TI + 4, kStrideB = kAlongB ? kDeep + 4 : TJ + 4;
  static constexpr int kFloatsA = kAlongA ? TI * kStrideA : kDeep * kStrideA, kFloatsB = kAlongB ? TJ * kStrideB : kDeep * kStrideB;
  static constexpr int kBuffer = kFloatsA + kSets * kFloatsB, kBuffers = sizeof(T) == 4 ? 4 : 2, kPad = TJ + 4;
  static constexpr int kFloats = kSets * TI * kPad > kBuffers * kBuffer ? kSets * TI * kPad : kBuffers * kBuffer;
  // row (column) i of a thread: every kLanesI-th (kLanesJ-th) along, four neighbours at a time across
  static __device__ __forceinline__ int row(int ty, int i) { return kAlongA ? ty + kLanesI * i : 4 * ty + 4 * kLanesI * (i / 4) + i % 4; }
  static __device__ __forceinline__ int col(int tx, int j) { return kAlongB ? tx + kLanesJ * j : 4 * tx + 4 * kLanesJ * (j / 4) + j % 4; }
};

__device__ __forceinline__ float2 fma_2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*(uint64_t*)&r) : "l"(*(const uint64_t*)&a), "l"(*(const uint64_t*)&b), "l"(*(const uint64_t*)&c));
  return r;
}
__device__ __forceinline__ uint32_t cluster_ctas() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_place() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Eight floats at the place of `at` in another CTA's shared memory
__device__ __forceinline__ void load_of_cta(const float* at, int rank, float (&v)[8]) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(at)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(a) : "memory");
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(a + 16) : "memory");
}
// `count` floats (0 .. V) from memory, zeros behind them.
template <int V>
__device__ __forceinline__ void copy_floats(float* to, const float* from, int count) {
  if (V == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(4 * count) : "memory");
  else if (V == 2) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(4 * count) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(4 * count) : "memory");
}

// One thread's units (V elements each) of an operand's steps: ROWS of it, the reduction along (ALONG) or across its rows.  Its units have one column and
// every kRows-th row of the buffer, so that an address is an addition.
template <typename T, int ROWS, bool ALONG, int STRIDE, int THREADS, int V>
struct Part {
  static constexpr int kAcross = (ALONG ? kDeep : ROWS) / V, kRows = THREADS / kAcross, kEach = (ALONG ? ROWS : kDeep) / kRows;
  static_assert(THREADS % kAcross == 0 && kEach * kRows == (ALONG ? ROWS : kDeep), "whole units");
  const T* from;         // first unit of the next step
  int64_t ld, step;
  int r, c, rows;        // row and column of the first unit; rows (along) or columns (across) that exist
  // base: first row (along) or first of the reduction (across) of the tile, first column
  __device__ __forceinline__ Part(const T* base, int64_t ld_, int rows_) : ld(ld_), step(ALONG ? kDeep : kDeep * ld_), rows(rows_) {
    r = threadIdx.x / kAcross, c = threadIdx.x % kAcross * V;
    from = base + r * ld + c;
  }
  // elements of unit i that exist, `left` of the reduction being left
  __device__ __forceinline__ int count(int i, int left) const {
    const int a = ALONG ? left - c : rows - c, n = a < 0 ? 0 : a < V ? a : V;
    return r + i * kRows < (ALONG ? rows : left) ? n : 0;
  }
  __device__ __forceinline__ void copy(float* buffer, int left, const T* any) {
    float* to = buffer + r * STRIDE + c;
    const T* p = from;
#pragma unroll
    for (int i = 0; i < kEach; ++i, p += kRows * ld) {
      const int n = count(i, left);
      copy_floats<V>(to + i * kRows * STRIDE, n ? p : any, n);
    }
    from += step;
  }
  __device__ __forceinline__ void fetch(float (&v)[kEach], int left) {
    const T* p = from;
#pragma unroll
    for (int i = 0; i < kEach; ++i, p += kRows * ld) v[i] = count(i, left) ? load_as_float(p) : 0.f;
    from += step;
  }
  __device__ __forceinline__ void put(float* buffer, const float (&v)[kEach]) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) buffer[(r + i * kRows) * STRIDE + c] = v[i];
  }
};

template <Kind KIND, typename T, bool GATED, int V>
__global__ void __launch_bounds__(General<KIND, T, GATED>::kThreads, KIND == kForward && GATED ? 3 : 4) general_kernel(const Problem p) {
  typedef General<KIND, T, GATED> C;
  constexpr int kSets = C::kSets, kThreads = C::kThreads, TI = C::TI, TJ = C::TJ, kPad = C::kPad;
  extern __shared__ __align__(16) float smem[];
  after_previous();
  float* Cs = smem;   // [kSets][TI][kPad], after the products
  int* before = (int*)(smem + C::kFloats);
  int* scratch = before + p.groups.G + 1;
  // A warp has 8 x 4 of the threads' places, and neighbouring lanes differ in both, so that any few lanes share what they read of either operand: 16-byte loads
  // from shared memory are served some lanes at a time.  16 groups of 256 rows x 2048 x 512: 264 -> 248 us, row gradient 258 -> 249, weight gradient
  // 232 -> 207 (five CTAs per SM, now four); the same 8 x 4 without neighbours in both gained nothing.
  const int t = threadIdx.x, tx = t / 2 % 8 + t / 32 % 2 * 8, ty = t % 2 + t / 16 % 2 * 2 + t / 64 * 4;
  static_assert(C::kLanesJ == 16 && C::kLanesI == 8, "the places of 128 threads");

  const int cols = KIND == kForward ? p.n : p.k;
  const int JT = (cols + TJ - 1) / TJ;
  int64_t items;
  const int IT = (p.n + TI - 1) / TI;               // kDweight: tiles of dout's columns
  constexpr int kHalves = KIND == kDweight && GATED ? 2 : 1;
  if (KIND == kDweight) {
    items = (int64_t)p.groups.G * kHalves * IT * JT;
  } else {
    count_tiles(p.groups, TI, before, scratch);
    items = (int64_t)before[p.groups.G] * JT;
  }
  const int ctas = (int)cluster_ctas(), place = (int)cluster_place();   // several CTAs on one tile share its reduction
  for (int64_t item = blockIdx.x / ctas; item < items; item += gridDim.x / ctas) {
    int g, i0, j0 = (int)(item % JT) * TJ, half = 0;
    if (KIND == kDweight) {
      int64_t r = item / JT;
      i0 = (int)(r % IT) * TI, r /= IT;
      half = (int)(r % kHalves), g = (int)(r / kHalves);
    } else {
      const int tile = (int)(item / JT);
      g = find_group(before, p.groups.G, tile);
      i0 = (tile - before[g]) * TI;
    }
    const GroupRows gr = group_rows(p.groups, g);
    const int64_t row0 = gr.first + (KIND == kDweight ? 0 : i0);
    const int I = KIND == kDweight ? min(TI, p.n - i0) : (int)min((int64_t)TI, gr.m - i0);
    const int J = min(TJ, cols - j0);
    const int red = KIND == kForward ? p.k : KIND == kBackward ? p.n : (int)gr.m;
    const int all_steps = red / kDeep + (red % kDeep != 0), each = (all_steps + ctas - 1) / ctas;
    const int first = min(place * each, all_steps), steps = min(first + each, all_steps) - first;   // this CTA's
    // Sums in pairs for the packed multiply-add: of the even and the odd products where both operands lie along, else of two neighbouring columns
    constexpr bool kByProduct = C::kAlongA && C::kAlongB;
    constexpr int kPairs = kByProduct ? C::RJ : C::RJ / 2;
    float2 c[kSets][C::RI][kPairs] = {};
    auto multiply = [&](const float* A) {
      const float* B = A + C::kFloatsA;
#pragma unroll
      for (int d = 0; d < kDeep; d += 4) {
        float a[C::RI][4];   // [row][product]
#pragma unroll
        for (int i = 0; i < C::RI; ++i) {
          const float4 v = *(const float4*)(C::kAlongA ? A + C::row(ty, i) * C::kStrideA + d : A + (d + i) * C::kStrideA + C::row(ty, 0));
          if (C::kAlongA) a[i][0] = v.x, a[i][1] = v.y, a[i][2] = v.z, a[i][3] = v.w;
          else a[0][i] = v.x, a[1][i] = v.y, a[2][i] = v.z, a[3][i] = v.w;
        }
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
          for (int q = 0; q < 4; ++q) {   // along: column q; across: product d + q
            const float4 b = *(const float4*)(B + s * C::kFloatsB + (C::kAlongB ? C::col(tx, q) * C::kStrideB + d : (d + q) * C::kStrideB + C::col(tx, 0)));
#pragma unroll
            for (int i = 0; i < C::RI; ++i) {
              if (kByProduct) {
                c[s][i][q] = fma_2(make_float2(a[i][0], a[i][1]), make_float2(b.x, b.y), c[s][i][q]);
                c[s][i][q] = fma_2(make_float2(a[i][2], a[i][3]), make_float2(b.z, b.w), c[s][i][q]);
              } else {
                const float2 twice = make_float2(a[i][q], a[i][q]);
                c[s][i][0] = fma_2(twice, make_float2(b.x, b.y), c[s][i][0]);
                c[s][i][1] = fma_2(twice, make_float2(b.z, b.w), c[s][i][1]);
              }
            }
          }
      }
    };
    for (int part = 0; part < (KIND == kBackward && GATED ? 2 : 1); ++part) {
      const T *base_a, *base_b, *base_b2 = nullptr;
      int64_t ld_a, ld_b;
      if (KIND == kForward) {
        base_a = (const T*)p.x + row0 * p.ld_x, ld_a = p.ld_x;
        const int64_t at = g * p.step_w + (int64_t)j0 * p.ld_w;
        base_b = (const T*)p.w + at, ld_b = p.ld_w;
        if (kSets == 2) base_b2 = (const T*)p.w_up + at;
      } else if (KIND == kBackward) {
        base_a = (const T*)p.y + row0 * p.ld_y + part * p.half_y, ld_a = p.ld_y;
        base_b = (const T*)(part ? p.w_up : p.w) + g * p.step_w + j0, ld_b = p.ld_w;
      } else {
        base_a = (const T*)p.y + gr.first * p.ld_y + half * p.half_y + i0, ld_a = p.ld_y;
        base_b = (const T*)p.x + gr.first * p.ld_x + j0, ld_b = p.ld_x;
      }
      const int64_t skip = (int64_t)first * kDeep;
      const int mine = red - first * kDeep;
      Part<T, TI, C::kAlongA, C::kStrideA, kThreads, V> pa(base_a + skip * (C::kAlongA ? 1 : ld_a), ld_a, I);
      typedef Part<T, TJ, C::kAlongB, C::kStrideB, kThreads, V> PartB;
      auto left_of = [&](int step) { return min(mine - step * kDeep, kDeep); };
      const int64_t skip_b = skip * (C::kAlongB ? 1 : ld_b);
      PartB pb(base_b + skip_b, ld_b, J), pb2((kSets == 2 ? base_b2 : base_b) + skip_b, ld_b, J);
      if constexpr (sizeof(T) == 4) {
        auto ask = [&](int step) {
          if (step < steps) {
            float* buffer = smem + step % C::kBuffers * C::kBuffer;
            pa.copy(buffer, left_of(step), base_a), pb.copy(buffer + C::kFloatsA, left_of(step), base_a);
            if (kSets == 2) pb2.copy(buffer + C::kFloatsA + C::kFloatsB, left_of(step), base_a);
          }
          asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < C::kBuffers - 1; ++i) ask(i);
        for (int step = 0; step < steps; ++step) {
          asm volatile("cp.async.wait_group %0;" ::"n"(C::kBuffers - 2) : "memory");
          __syncthreads();   // everybody's copies of this step are there, and nobody reads the buffer that the next copies go to
          ask(step + C::kBuffers - 1);
          multiply(smem + step % C::kBuffers * C::kBuffer);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
      } else {
        float ra[decltype(pa)::kEach], rb[kSets][PartB::kEach];
        auto fetch = [&](int step) {
          pa.fetch(ra, left_of(step)), pb.fetch(rb[0], left_of(step));
          if (kSets == 2) pb2.fetch(rb[kSets - 1], left_of(step));
        };
        auto put = [&](int step) {
          float* buffer = smem + step % C::kBuffers * C::kBuffer;
          pa.put(buffer, ra), pb.put(buffer + C::kFloatsA, rb[0]);
          if (kSets == 2) pb2.put(buffer + C::kFloatsA + C::kFloatsB, rb[kSets - 1]);
        };
        if (steps) fetch(0), put(0);
        __syncthreads();
        for (int step = 0; step < steps; ++step) {
          if (step + 1 < steps) fetch(step + 1);
          multiply(smem + step % C::kBuffers * C::kBuffer);
          if (step + 1 < steps) put(step + 1);
          __syncthreads();
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < C::RI; ++i)
#pragma unroll
        for (int j = 0; j < C::RJ; ++j)
          Cs[(s * TI + C::row(ty, i)) * kPad + C::col(tx, j)] = kByProduct ? c[s][i][j].x + c[s][i][j].y : j & 1 ? c[s][i][j / 2].y : c[s][i][j / 2].x;
    if (ctas > 1) cluster_wait();
    else __syncthreads();
    // Blocks of 8 rows x 32 columns, dealt to the warps of all CTAs of the tile.  What the CTAs hold of a result is added in the order of their ranks.
    auto sums_at = [&](int s, int i, int j, float (&v)[8]) {
      const float* at = Cs + (s * TI + i) * kPad + j;
      if (ctas == 1) {
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = at[u];
        return;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = 0.f;
      for (int r = 0; r < ctas; ++r) {
        float w[8];
        load_of_cta(at, r, w);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] += w[u];
      }
    };
    const int lane = t % 32;
    for (int block = place + ctas * (t / 32); block < TI / 8 * (TJ / 32); block += ctas * (kThreads / 32)) {
      const int jj = block % (TJ / 32) * 32, ii = block / (TJ / 32) * 8;
      if (jj >= J || ii >= I) continue;
      const int i = ii + lane / 4, j = jj + 8 * (lane % 4);
      float z[1][8], up[1][8] = {};
      sums_at(0, i, j, z[0]);
      if (kSets == 2) sums_at(1, i, j, up[0]);
      if constexpr (KIND == kDweight) {
        const int count = i < I ? min(max(J - j, 0), 8) : 0;
        const void* add = half ? p.add_dw_up : p.add_dw;
        void* dw = half ? p.dw_up : p.dw;
        const int64_t at = g * p.step_w + (int64_t)(i0 + i) * p.ld_w + j0 + j;
        auto finish = [&](auto* o, const auto* from) {
          if (!count) return;
          if (from) {
            uint32_t w[2 * sizeof(*o)];
            float v[8];
            load_8(from, p.dw_wide == 2, count, w);
            floats_of(w, v);
#pragma unroll
            for (int u = 0; u < 8; ++u) z[0][u] += v[u];
          }
          store_8(o, p.dw_wide == 2, count, z[0]);
        };
        if (p.dw_f32) finish((float*)dw + at, add ? (const float*)add + at : nullptr);
        else finish((T*)dw + at, add ? (const T*)add + at : nullptr);
      } else if constexpr (KIND == kForward) {
        const Forward<T, GATED> e(p.fwd, g, j0 + j);
        e.rows(row0 + ii, I - ii, z, up);
      } else {
        const Backward<T> e(p.bwd, g, j0 + j);
        typename Backward<T>::template Asked<1> q;
        e.ask(row0 + ii, I - ii, q);
        e.rows(row0 + ii, I - ii, z, q);
      }
    }
    if (ctas > 1) cluster_wait();
    else __syncthreads();
  }
}

// Tiles of a product, at most
constexpr int kTileI = 32, kTileJ = 64;
int64_t general_tiles(Kind kind, const Problem& p) {
  const int64_t across = ((kind == kForward ? p.n : p.k) + kTileJ - 1) / kTileJ;
  if (kind == kDweight) return (int64_t)p.groups.G * (p.gated ? 2 : 1) * ((p.n + kTileI - 1) / kTileI) * across;
  return (p.L * p.groups.R / kTileI + p.groups.G) * across;
}
int64_t reduction(Kind kind, const Problem& p) { return kind == kForward ? p.k : kind == kBackward ? p.n : p.L * p.groups.R / p.groups.G; }
// CTAs per tile: as many as make six CTAs per SM in all and leave each of them eight steps.  Four (a gated forward pass: three) are on an SM at once; the others
// take the places of those that are done, where a limit of three or four often leaves whole SMs without a second one.  fp32, rows / groups x k x n, us with one CTA
// per tile / up to three / four / six / eight per SM:
//   900/10 x 1002 x 515: 58 / 58 / 58 / 50 / 50     2000/16 x 640 x 256: 34 / 34 / 34 / 25 / 25     1024/4 x 1024 x 512: 36 / 36 / 37 / 37 / 39
//   4/30 x 2034 x 64: 50 / 10 / 10 / 10 / 10        512/8 x 2048 x 512: 67 / 53 / 53 / 45 / 45     64/8 x 2048 x 512, gated: 77 / 37 / 37 / 43 / 43
int general_ctas(Kind kind, const Problem& p, int64_t tiles, int sms) {
  int ctas = 8;
  while (ctas > 1 && (tiles * ctas > 6 * sms || reduction(kind, p) < 8 * kDeep * ctas)) ctas /= 2;
  return ctas;
}

template <Kind KIND, typename T, bool GATED, int V>
cudaError_t launch_tiles(const Problem& p, int64_t tiles, int sms, cudaStream_t st) {
  static int cache[64] = {0};
  constexpr size_t kBytes = General<KIND, T, GATED>::kFloats * 4;
  const cudaError_t e = tc::sm_count_and_smem_optin(general_kernel<KIND, T, GATED, V>, kBytes + (MCCE_LINEAR_MAX_GROUPS + 1 + 33) * 4, cache, &sms);
  if (e != cudaSuccess) return e;
  const int ctas = general_ctas(KIND, p, tiles, sms);
  const int64_t most = 8 * sms / ctas;
  return launch_close(general_kernel<KIND, T, GATED, V>, dim3((unsigned)((tiles < most ? tiles : most) * ctas)), General<KIND, T, GATED>::kThreads,
                      kBytes + (size_t)(p.groups.G + 1 + 33) * 4, st, ctas, p);
}
template <Kind KIND, typename T, bool GATED, int V>
cudaError_t launch_general(const Problem& p, cudaStream_t st) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaErrorInvalidDevice;
  static_assert(General<KIND, T, GATED>::TI == kTileI && General<KIND, T, GATED>::TJ == kTileJ, "the tiles that are counted");
  return launch_tiles<KIND, T, GATED, V>(p, general_tiles(KIND, p), sms, st);
}
template <Kind KIND, typename T, int V>
cudaError_t launch_general_gated(const Problem& p, cudaStream_t st) {
  return p.gated ? launch_general<KIND, T, true, V>(p, st) : launch_general<KIND, T, false, V>(p, st);
}
template <Kind KIND>
cudaError_t launch_general_types(const Problem& p, int32_t dtype, cudaStream_t st) {
  if (dtype == MCCE_BF16) return launch_general_gated<KIND, __nv_bfloat16, 1>(p, st);
  auto aligned_to = [&](int v) {   // v columns of what this product reads: x and the weights, dout and the weights, dout and x
    auto one = [&](const void* a, int64_t ld) { return !a || (((uintptr_t)a | (uintptr_t)(ld * 4)) & (4 * v - 1)) == 0; };
    return (KIND == kBackward || one(p.x, p.ld_x)) && (KIND == kForward || (one(p.y, p.ld_y) && (!p.gated || p.half_y % v == 0))) &&
           (KIND == kDweight || (one(p.w, p.ld_w) && one(p.w_up, p.ld_w) && (p.groups.G == 1 || p.step_w % v == 0)));
  };
  if (aligned_to(4)) return launch_general_gated<KIND, float, 4>(p, st);
  return aligned_to(2) ? launch_general_gated<KIND, float, 2>(p, st) : launch_general_gated<KIND, float, 1>(p, st);
}

// ---- sums of dout's columns per group (the bias's gradient) ----------------------------------------------------
struct BiasArgs {
  Groups groups;
  int32_t n, gated, f32, wide, chunks;
  int64_t ld_y, half_y;
  const void *y, *add, *add_up;
  void *db, *db_up;
  float* parts;   // [chunks][halves][G][n], null with one chunk
};
template <typename T>
__device__ __forceinline__ void bias_store(const BiasArgs& a, int half, int64_t at, float v) {
  const void* add = half ? a.add_up : a.add;
  void* db = half ? a.db_up : a.db;
  if (a.f32) ((float*)db)[at] = v + (add ? ((const float*)add)[at] : 0.f);
  else store_as((T*)db + at, v + (add ? load_as_float((const T*)add + at) : 0.f));
}
// A CTA of 8 warps sums 256 columns (eight per lane) of one group, or of one chunk of its rows; a warp takes every eighth row, four under way.  Parts
// are added in a fixed order.
template <typename T>
__global__ void __launch_bounds__(256) bias_kernel(const BiasArgs a) {
  __shared__ float part[8][256 + 8];
  after_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = blockIdx.y, half = blockIdx.z % (a.gated + 1), chunk = blockIdx.z / (a.gated + 1);
  const int j = blockIdx.x * 256 + 8 * lane, count = min(max(a.n - j, 0), 8);
  const GroupRows gr = group_rows(a.groups, g);
  const int64_t each = (gr.m + a.chunks - 1) / a.chunks, lo = min(chunk * each, gr.m), hi = min(lo + each, gr.m);
  const T* y = (const T*)a.y + gr.first * a.ld_y + half * a.half_y + j;
  float s[8] = {};
  if (count)
    for (int64_t r = lo + warp; r < hi; r += 32) {
      uint32_t w[4][2 * sizeof(T)];
#pragma unroll
      for (int u = 0; u < 4; ++u) load_8(y + min(r + 8 * u, hi - 1) * a.ld_y, a.wide, count, w[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float v[8];
        floats_of(w[u], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += r + 8 * u < hi ? v[i] : 0.f;
      }
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[warp][8 * lane + i] = s[i];
  __syncthreads();
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) v += part[w][threadIdx.x];
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= a.n) return;
  const int64_t at = (int64_t)g * a.n + col;
  if (a.parts) {
    a.parts[(int64_t)(chunk * (a.gated + 1) + half) * a.groups.G * a.n + at] = v;
    return;
  }
  bias_store<T>(a, half, at, v);
}
template <typename T>
__global__ void __launch_bounds__(256) bias_parts_kernel(const BiasArgs a) {
  const int64_t at = blockIdx.x * 256ll + threadIdx.x, all = (int64_t)a.groups.G * a.n;
  after_previous();
  if (at >= all) return;
  float v = 0.f;
  for (int c = 0; c < a.chunks; ++c) v += a.parts[(int64_t)(c * (a.gated + 1) + blockIdx.y) * all + at];
  bias_store<T>(a, blockIdx.y, at, v);
}

// ---- 8-bit checkpoints ------------------------------------------------------------------------------------------
// Rows whose columns are aligned eight at a time: four lanes have a block of 32 columns, and a lane has U blocks, kStride blocks apart, under way.
// 16384 x 4096 bf16: two blocks 39.5 us, one 47, four 48, eight 64 (bound by instructions; fp32, 8192 rows: 27 us, HBM).
template <typename T, int U>
__global__ void __launch_bounds__(256) pack_kernel(const T* x, uint8_t* q, uint8_t* scales, int64_t blocks, int per_row, int d, int64_t ld_x,
                                                   int64_t ld_q) {
  const int64_t first = (int64_t)blockIdx.x * (64 * U) + threadIdx.x / 4;
  after_previous();
  uint32_t raw[U][2 * sizeof(T)];
  int count[U], col[U];
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t b = min(first + 64 * u, blocks - 1);
    row[u] = (uint32_t)(b >> 32) ? b / per_row : (uint32_t)b / (uint32_t)per_row;
    col[u] = (int)(b - row[u] * per_row) * 32 + 8 * (threadIdx.x & 3), count[u] = min(max(d - col[u], 0), 8);
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) raw[u][i] = 0u;
    if (count[u]) load_8(x + row[u] * ld_x + col[u], true, count[u], raw[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[8];
    uint32_t w[2];
    floats_of(raw[u], v);
    const uint32_t s = pack_8(v, largest_bits(raw[u]), w);
    const int64_t b = first + 64 * u;
    if (b >= blocks) continue;
    if (count[u]) store_words_8(q + row[u] * ld_q + col[u], true, count[u], w);
    if ((threadIdx.x & 3) == 0) scales[b] = (uint8_t)s;
  }
}
template <typename T, int U>
__global__ void __launch_bounds__(256) unpack_kernel(const uint8_t* q, const uint8_t* scales, T* x, int64_t blocks, int per_row, int d,
                                                     int64_t ld_x, int64_t ld_q) {
  const int64_t first = (int64_t)blockIdx.x * (64 * U) + threadIdx.x / 4;
  after_previous();
  uint32_t w[U][2], s[U];
  int count[U], col[U];
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t b = min(first + 64 * u, blocks - 1);
    row[u] = (uint32_t)(b >> 32) ? b / per_row : (uint32_t)b / (uint32_t)per_row;
    col[u] = (int)(b - row[u] * per_row) * 32 + 8 * (threadIdx.x & 3), count[u] = first + 64 * u < blocks ? min(max(d - col[u], 0), 8) : 0;
    w[u][0] = w[u][1] = 0u;
    if (count[u]) load_8(q + row[u] * ld_q + col[u], true, count[u], w[u]);
    s[u] = scales[b];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[8];
    floats_of(w[u], v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= scale_value(s[u]);
    if (count[u]) store_8(x + row[u] * ld_x + col[u], true, count[u], v);
  }
}
// Any other rows: a column per lane, a warp takes eight blocks of a row at a time.
template <typename T>
__global__ void __launch_bounds__(256) pack_odd_kernel(const T* x, uint8_t* q, uint8_t* scales, int64_t rows, int per_row, int d, int64_t ld_x,
                                                       int64_t ld_q) {
  const int lane = threadIdx.x & 31, parts = (per_row + 7) / 8;
  after_previous();
  const int64_t w = blockIdx.x * 8ll + (threadIdx.x >> 5), row = w / parts;
  if (row >= rows) return;
  const int b0 = (int)(w - row * parts) * 8;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (b0 + i) * 32 + lane < d ? load_as_float(x + row * ld_x + (b0 + i) * 32 + lane) : 0.f;
  uint32_t mine = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t s = warp_block_scale(v[i]);
    if ((b0 + i) * 32 + lane < d) q[row * ld_q + (b0 + i) * 32 + lane] = (uint8_t)to_e4m3x2(v[i] * scale_inverse(s), 0.f);
    if (lane == i) mine = s;
  }
  if (lane < 8 && b0 + lane < per_row) scales[row * per_row + b0 + lane] = (uint8_t)mine;
}
template <typename T>
__global__ void __launch_bounds__(256) unpack_odd_kernel(const uint8_t* q, const uint8_t* scales, T* x, int64_t rows, int per_row, int d,
                                                         int64_t ld_x, int64_t ld_q) {
  const int lane = threadIdx.x & 31, parts = (per_row + 7) / 8;
  after_previous();
  const int64_t w = blockIdx.x * 8ll + (threadIdx.x >> 5), row = w / parts;
  if (row >= rows) return;
  const int b0 = (int)(w - row * parts) * 8;
  uint32_t v[8];
  const uint32_t s = b0 + (lane & 7) < per_row ? scales[row * per_row + b0 + (lane & 7)] : 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (b0 + i) * 32 + lane < d ? q[row * ld_q + (b0 + i) * 32 + lane] : 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = e4m3x2_value(v[i]).x * scale_value(__shfl_sync(0xffffffffu, s, i));
    if ((b0 + i) * 32 + lane < d) store_as(x + row * ld_x + (b0 + i) * 32 + lane, f);
  }
}

}  // namespace

cudaError_t run_general(Kind kind, const Problem& p, int32_t dtype, cudaStream_t st) {
  if (kind == kForward) return launch_general_types<kForward>(p, dtype, st);
  return kind == kBackward ? launch_general_types<kBackward>(p, dtype, st) : launch_general_types<kDweight>(p, dtype, st);
}

namespace {
// Eight columns of every row start at a multiple of what they take, 16 bytes at most.
bool wide_rows(const void* p, int64_t ld, int e) { return !p || (((uintptr_t)p | (uintptr_t)(ld * e)) & (e == 1 ? 7 : 15)) == 0; }
}  // namespace

// Chunks of a group's rows: one unless the groups are few and long; up to four CTAs for each of a B200's 148 SMs, each with 512 rows or more.  (The workspace
// is asked for without a device, so that this goes by the SMs that the library is built for; so do the copies below and the blocks per lane of a checkpoint.)
int bias_chunks(int64_t rows, int32_t G, int32_t n) {
  constexpr int64_t kMost = 4 * 148;
  const int64_t ctas = (int64_t)G * ((n + 255) / 256), each = rows / G / 512;
  if (each < 2 || ctas >= kMost) return 1;
  const int64_t want = kMost / ctas;
  return (int)(each < want ? each : want < 64 ? want : 64);
}
cudaError_t run_bias_sums(const Problem& p, int32_t dtype, const void* add, const void* add_up, void* db, void* db_up, float* parts,
                          cudaStream_t st) {
  const int halves = p.gated ? 2 : 1, e = dtype == MCCE_F32 ? 4 : 2, chunks = bias_chunks(p.L * p.groups.R, p.groups.G, p.n);
  const bool wide = wide_rows(p.y, p.ld_y, e) && (!p.gated || p.half_y * e % 16 == 0);
  const BiasArgs a{p.groups, p.n, p.gated, p.dw_f32, wide, chunks, p.ld_y, p.half_y, p.y, add, add_up, db, db_up, chunks > 1 ? parts : nullptr};
  const dim3 grid((p.n + 255) / 256, p.groups.G, halves * chunks), all((unsigned)(((int64_t)p.groups.G * p.n + 255) / 256), halves);
  const cudaError_t err = dtype == MCCE_F32 ? launch_close(bias_kernel<float>, grid, 256, 0, st, 1, a)
                                            : launch_close(bias_kernel<__nv_bfloat16>, grid, 256, 0, st, 1, a);
  if (err != cudaSuccess || chunks == 1) return err;
  return dtype == MCCE_F32 ? launch_close(bias_parts_kernel<float>, all, 256, 0, st, 1, a)
                           : launch_close(bias_parts_kernel<__nv_bfloat16>, all, 256, 0, st, 1, a);
}

namespace {
template <typename T>
cudaError_t pack_as(bool pack, const void* x, void* to, const uint8_t* q_in, uint8_t* q, const uint8_t* s_in, uint8_t* scales, int64_t rows, int32_t d,
                    int64_t ld_x, int64_t ld_q, cudaStream_t st) {
  const int per_row = (d + 31) / 32;
  const bool wide = pack ? wide_rows(x, ld_x, sizeof(T)) && wide_rows(q, ld_q, 1) : wide_rows(to, ld_x, sizeof(T)) && wide_rows(q_in, ld_q, 1);
  const int64_t blocks = rows * per_row;
  constexpr int kU = 2;
  const bool many = blocks >= 148 * 8 * 64 * kU;   // else one block per lane: more CTAs
  const int64_t grid = !wide ? (rows * ((per_row + 7) / 8) + 7) / 8 : many ? (blocks + 64 * kU - 1) / (64 * kU) : (blocks + 63) / 64;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  const dim3 n((unsigned)grid);
  if (pack) {
    const T* from = (const T*)x;
    if (!wide) return launch_close(pack_odd_kernel<T>, n, 256, 0, st, 1, from, q, scales, rows, per_row, d, ld_x, ld_q);
    return launch_close(many ? pack_kernel<T, kU> : pack_kernel<T, 1>, n, 256, 0, st, 1, from, q, scales, blocks, per_row, d, ld_x, ld_q);
  }
  if (!wide) return launch_close(unpack_odd_kernel<T>, n, 256, 0, st, 1, q_in, s_in, (T*)to, rows, per_row, d, ld_x, ld_q);
  return launch_close(many ? unpack_kernel<T, kU> : unpack_kernel<T, 1>, n, 256, 0, st, 1, q_in, s_in, (T*)to, blocks, per_row, d, ld_x, ld_q);
}
}  // namespace

cudaError_t run_pack(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, uint8_t* q, uint8_t* scales,
                     cudaStream_t st) {
  return dtype == MCCE_F32 ? pack_as<float>(true, x, nullptr, nullptr, q, nullptr, scales, rows, d, ld_x, ld_q, st)
                           : pack_as<__nv_bfloat16>(true, x, nullptr, nullptr, q, nullptr, scales, rows, d, ld_x, ld_q, st);
}
cudaError_t run_unpack(const uint8_t* q, const uint8_t* scales, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, void* x,
                       cudaStream_t st) {
  return dtype == MCCE_F32 ? pack_as<float>(false, nullptr, x, q, nullptr, scales, nullptr, rows, d, ld_x, ld_q, st)
                           : pack_as<__nv_bfloat16>(false, nullptr, x, q, nullptr, scales, nullptr, rows, d, ld_x, ld_q, st);
}

// ---- bf16 rows to strides and starts of 16 bytes ------------------------------------------------------------------
namespace {
// Eight elements per lane, read as words (of a start between two words: five, shifted), the last of a row one by one.  Row r is row r % per of matrix r / per.
__global__ void __launch_bounds__(256) align_kernel(const uint16_t* from, int64_t units, int64_t per, int cols, int across, int64_t ld, int64_t step,
                                                    uint16_t* to, int64_t ld_to) {
  after_previous();
  const int64_t u = blockIdx.x * 256ll + threadIdx.x;
  if (u >= units) return;
  const int64_t row = u / across;
  const int c = (int)(u - row * across) * 8;
  const uint16_t* p = from + row / per * step + row % per * ld + c;
  uint32_t w[4] = {};
  if (c + 9 <= cols) {
    const uint32_t* a = (const uint32_t*)((uintptr_t)p & ~(uintptr_t)3);
    if ((uintptr_t)p & 2) {
      uint32_t v[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) v[i] = a[i];   // the element before the eight and the one behind them are the row's or, before its first, its word's
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = a[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
  }
  *(uint4*)(to + row * ld_to + c) = make_uint4(w[0], w[1], w[2], w[3]);
}
}  // namespace
cudaError_t run_align(const void* from, int64_t rows, int64_t per, int32_t cols, int64_t ld, int64_t step, void* to, int64_t ld_to, cudaStream_t st) {
  const int across = (cols + 7) / 8;
  const int64_t units = rows * across, grid = (units + 255) / 256;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_close(align_kernel, dim3((unsigned)grid), 256, 0, st, 1, (const uint16_t*)from, units, per, cols, across, ld, step, (uint16_t*)to, ld_to);
}

// ---- checks --------------------------------------------------------------------------------------------------------
namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
int elem(int32_t dtype) { return dtype == MCCE_F32 ? 4 : dtype == MCCE_BF16 ? 2 : 1; }
bool plain_type(int32_t t) { return t == MCCE_F32 || t == MCCE_BF16; }
int64_t ld_or(int64_t ld, int64_t d) { return ld ? ld : d; }
bool stride_ok(int64_t ld, int64_t d) { return ld == 0 || ld >= d; }

bool sizes_ok(const mcce_linear* p) {
  if (!p || p->n_layers < 1 || p->n_experts < 1 || (int64_t)p->n_layers * p->n_experts > MCCE_LINEAR_MAX_GROUPS) return false;
  if (p->rows < 0 || p->rows > 0x7fffffffll || p->n_layers * p->rows > 0x7fffffffll) return false;
  if (p->n < 1 || p->k < 1 || p->n > MCCE_LINEAR_MAX_WIDTH || p->k > MCCE_LINEAR_MAX_WIDTH) return false;
  if (!plain_type(p->dtype) || (p->gated != 0 && p->gated != 1)) return false;
  if (!stride_ok(p->ld_w, p->k)) return false;
  const int64_t ld_w = ld_or(p->ld_w, p->k);
  if (ld_w > (1ll << 40) || (p->step_w != 0 && p->step_w < (p->n - 1) * ld_w + p->k) || p->step_w > (1ll << 48)) return false;
  return true;
}
bool act_ok(int32_t act) { return act == MCCE_ACT_NONE || act == MCCE_ACT_SILU || act == MCCE_ACT_GELU; }

// All rows of the weights for the comparison of addresses
Span weight_span(const mcce_linear& p, const void* w, int e) {
  const int64_t ld = ld_or(p.ld_w, p.k), step = p.step_w ? p.step_w : p.n * ld, G = (int64_t)p.n_layers * p.n_experts;
  if (step == p.n * ld || G == 1) return row_span(w, G * p.n, ld, p.k, e);
  if (ld == p.k) return row_span(w, G, step, p.n * ld, e);
  return stack_span(w, G, step, p.n, ld, p.k, e);
}
Problem problem(const mcce_linear& p, const int32_t* offsets) {
  Problem q{};
  q.groups = {offsets, p.n_experts, p.n_layers * p.n_experts, p.rows};
  q.n = p.n, q.k = p.k, q.gated = p.gated, q.L = p.n_layers, q.half_y = p.n;
  q.ld_w = ld_or(p.ld_w, p.k), q.step_w = p.step_w ? p.step_w : p.n * q.ld_w;
  return q;
}
int blocks_of(int64_t cols) { return (int)((cols + 31) / 32); }
int code(cudaError_t e) { return e == cudaSuccess ? MCCE_OK : MCCE_ECUDA; }

// bf16 rows that the tensor cores' copies cannot take (a stride or start that is no multiple of 16 bytes) are brought to one that is, where that pays: on the fp32
// pipe bf16 products run at 10 to 20 TFLOP/s (4096 x 2047 x 511, gated: 800 us, copied 74), the copies at some 4 TB/s.
// Both ways were timed over 396 products (forward, row and weight gradient, gated and not, 64 to 65536 rows of 1 to 64 groups, widths 65 to 2050): the estimate takes
// the slower one by more than 12 % in 40 of them, and 5 % more than the faster ones in the mean.  Where it copies in vain that costs up to 9 us (weight gradient of
// 1024 rows x 255 x 255, gated: 15 -> 24); where it does not copy, gated row gradients of few rows lose most (64 rows x 255 x 255: 18 -> 73 us; they
// run at a quarter of the others' rate).  With the time of a weight gradient's slabs, which a pair of CTAs takes one after the other, in the estimate it was 48 of 396.
struct Copies {
  bool x, y, w;
  size_t x_bytes, y_bytes, w_bytes;   // w: of one matrix of every group
  size_t bytes(bool gated) const { return x_bytes + y_bytes + (gated ? 2 : 1) * w_bytes; }
};
int64_t whole_8(int64_t cols) { return (cols + 7) & ~7ll; }
Copies copies_for(Kind kind, const Problem& q, int32_t dtype) {
  Copies c{};
  if (dtype != MCCE_BF16 || tensor_applicable(kind, q, dtype)) return c;
  auto fits = [](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; };
  const int64_t rows = q.L * q.groups.R, G = q.groups.G;
  const int two = q.gated ? 2 : 1;
  c.x = kind != kBackward && !fits(q.x, q.ld_x);
  c.y = kind != kForward && !(fits(q.y, q.ld_y) && (!q.gated || q.half_y % 8 == 0));
  c.w = kind != kDweight && !(fits(q.w, q.ld_w) && fits(q.w_up, q.ld_w) && (G == 1 || q.step_w % 8 == 0));
  auto size = [](int64_t r, int64_t cols) { return ((size_t)r * cols * 2 + 255) & ~(size_t)255; };
  if (c.x) c.x_bytes = size(rows, whole_8(q.k));
  if (c.y) c.y_bytes = size(rows, two * whole_8(q.n));
  if (c.w) c.w_bytes = size(G * q.n, whole_8(q.k));
  if (rows == 0) return Copies{};
  // the fp32 pipe: its rate, and 0.4 us for every step of a CTA; the tensor cores: the copies, and their launches with the product's shortest time
  const double steps = (double)reduction(kind, q) / kDeep / general_ctas(kind, q, general_tiles(kind, q), 148);
  const double pipe = 2.0 * rows * q.n * q.k * two / 12e12 + steps * 0.4e-6, tensor = c.bytes(q.gated) * 2.0 / 4e12 + 22e-6;
  return pipe > tensor ? c : Copies{};
}
// Copies in front of a product: q then names them.
cudaError_t run_copies(const Copies& c, Problem& q, void* workspace, cudaStream_t st) {
  uint8_t* to = (uint8_t*)workspace;
  const int64_t rows = q.L * q.groups.R, k8 = whole_8(q.k), n8 = whole_8(q.n);
  cudaError_t err = cudaSuccess;
  if (c.x) {
    err = run_align(q.x, rows, rows, q.k, q.ld_x, 0, to, k8, st);
    q.x = to, q.ld_x = k8, to += c.x_bytes;
  }
  if (c.y) {
    for (int h = 0; h < (q.gated ? 2 : 1) && err == cudaSuccess; ++h)
      err = run_align((const __nv_bfloat16*)q.y + h * q.half_y, rows, rows, q.n, q.ld_y, 0, (__nv_bfloat16*)to + h * n8, (q.gated ? 2 : 1) * n8, st);
    q.y = to, q.ld_y = (q.gated ? 2 : 1) * n8, q.half_y = n8, to += c.y_bytes;
  }
  if (c.w) {
    for (int h = 0; h < (q.gated ? 2 : 1) && err == cudaSuccess; ++h) {
      const void*& w = h ? q.w_up : q.w;
      err = run_align(w, (int64_t)q.groups.G * q.n, q.n, q.k, q.ld_w, q.step_w, to, k8, st);
      w = to, to += c.w_bytes;
    }
    q.ld_w = k8, q.step_w = (int64_t)q.n * k8;
  }
  return err;
}
cudaError_t run_product(Kind kind, Problem& q, int32_t dtype, void* workspace, cudaStream_t st) {
  const Copies c = copies_for(kind, q, dtype);
  if (c.bytes(q.gated)) {
    const cudaError_t err = run_copies(c, q, workspace, st);
    if (err != cudaSuccess) return err;
  }
  if (kind == kForward && few_applicable(q, dtype)) return run_few(q, st);
  return tensor_applicable(kind, q, dtype) ? run_tensor(kind, q, st) : run_general(kind, q, dtype, st);
}

// Workspace of the weight gradient: 8-bit rows in the type of dout, then the parts of the bias's gradient.
size_t unpacked_bytes(const mcce_linear& p) {
  if (p.saved_dtype != MCCE_E4M3) return 0;
  const int64_t ld = (p.k + 7) & ~7ll;
  return ((size_t)(p.n_layers * p.rows) * ld * elem(p.dtype) + 255) & ~(size_t)255;
}
size_t bias_bytes(const mcce_linear& p) {
  const int32_t G = p.n_layers * p.n_experts;
  const int chunks = bias_chunks(p.n_layers * p.rows, G, p.n);
  return chunks > 1 ? ((size_t)chunks * (1 + p.gated) * G * p.n * 4 + 255) & ~(size_t)255 : 0;
}

// dout and x as the products see them: 8-bit x is unpacked to rows of whole 16 bytes first
Problem dweight_problem(const mcce_linear& p, const void* dout, const void* x) {
  Problem q = problem(p, nullptr);
  q.y = dout, q.ld_y = ld_or(p.ld_y, (int64_t)p.n * (1 + p.gated)), q.x = x, q.ld_x = ld_or(p.ld_x, p.k);
  if (p.saved_dtype == MCCE_E4M3) q.x = nullptr, q.ld_x = whole_8(p.k);
  return q;
}

}  // namespace
}  // namespace linear
}  // namespace mcce

using namespace mcce;
using namespace mcce::linear;

extern "C" int mcce_expert_linear(const mcce_linear* p, const void* x, const int32_t* offsets, const void* w, const void* w_up,
                                  const void* bias, const void* bias_up, const void* add, void* out, void* saved, void* scales,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(p) || !act_ok(p->act)) return MCCE_EINVAL;
  const int64_t width = (int64_t)p->n * (1 + p->gated), rows = p->n_layers * p->rows;
  if (p->out_dtype != MCCE_F32 && p->out_dtype != p->dtype) return MCCE_EINVAL;
  if (bias && p->bias_dtype != MCCE_F32 && p->bias_dtype != p->dtype) return MCCE_EINVAL;
  if (saved && p->saved_dtype != p->dtype && p->saved_dtype != MCCE_E4M3) return MCCE_EINVAL;
  const bool bytes = saved && p->saved_dtype == MCCE_E4M3;
  if (!stride_ok(p->ld_x, p->k) || !stride_ok(p->ld_y, p->n) || (add && !stride_ok(p->ld_add, p->n)) ||
      (saved && !stride_ok(p->ld_saved, width)))
    return MCCE_EINVAL;
  if ((w_up != nullptr) != (p->gated == 1) || (bias_up != nullptr) != (bias != nullptr && p->gated) || (scales != nullptr) != bytes)
    return MCCE_EINVAL;
  if (rows == 0) return MCCE_OK;
  if (!x || !offsets || !w || !out) return MCCE_EINVAL;
  const int e = elem(p->dtype), eo = elem(p->out_dtype), eb = elem(p->bias_dtype), es = bytes ? 1 : e;
  if (!aligned(x, e) || !aligned(offsets, 4) || !aligned(w, e) || !aligned(w_up, e) || (bias && (!aligned(bias, eb) || !aligned(bias_up, eb))) ||
      !aligned(add, eo) || !aligned(out, eo) || !aligned(saved, es))
    return MCCE_EINVAL;
  Problem q = problem(*p, offsets);
  q.x = x, q.w = w, q.w_up = w_up;
  q.ld_x = ld_or(p->ld_x, p->k);
  ForwardArgs& f = q.fwd;
  f.bias = bias, f.bias_up = bias_up, f.add = add, f.out = out, f.saved = saved, f.scales = (uint8_t*)scales;
  f.ld_add = ld_or(p->ld_add, p->n), f.ld_out = ld_or(p->ld_y, p->n), f.ld_saved = ld_or(p->ld_saved, width);
  f.bias_f32 = p->bias_dtype == MCCE_F32, f.out_f32 = p->out_dtype == MCCE_F32, f.act = p->act, f.n = p->n, f.blocks = blocks_of(p->n);
  f.wide = wide_rows(add, f.ld_add, eo) && wide_rows(out, f.ld_out, eo) && wide_rows(saved, f.ld_saved, es);
  const int64_t G = q.groups.G;
  const Span sx = row_span(x, rows, q.ld_x, p->k, e), soff = flat_span(offsets, (int64_t)p->n_layers * (p->n_experts + 1), 4);
  const Span sw = weight_span(*p, w, e), swu = weight_span(*p, w_up, e);
  const Span sb = flat_span(bias, G * p->n, eb), sbu = flat_span(bias_up, G * p->n, eb);
  const Span sadd = row_span(add, rows, f.ld_add, p->n, eo), sout = row_span(out, rows, f.ld_out, p->n, eo);
  const Span ssv = row_span(saved, rows, f.ld_saved, width, es), ssc = flat_span(scales, rows, (1 + p->gated) * (int64_t)f.blocks);
  const size_t need = copies_for(kForward, q, p->dtype).bytes(q.gated);
  if (need && (!workspace || !aligned(workspace, 16))) return MCCE_EINVAL;
  if (workspace_bytes < need) return MCCE_ENOSPC;
  const Span sws = flat_span(need ? workspace : nullptr, need);
  if (!same_or_apart(sout, sadd) || !apart(sout, {&sx, &soff, &sw, &swu, &sb, &sbu, &ssv, &ssc}) ||
      !apart(ssv, {&sx, &soff, &sw, &swu, &sb, &sbu, &sadd, &ssc}) || !apart(ssc, {&sx, &soff, &sw, &swu, &sb, &sbu, &sadd}) ||
      !apart(sws, {&sx, &soff, &sw, &swu, &sb, &sbu, &sadd, &sout, &ssv, &ssc}))
    return MCCE_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return code(run_product(kForward, q, p->dtype, workspace, st));
}

extern "C" int mcce_expert_linear_backward(const mcce_linear* p, const void* dout, const int32_t* offsets, const void* w,
                                           const void* w_up, const void* add, const void* saved, const void* scales, void* dx, void* h,
                                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(p) || !act_ok(p->act) || p->below < 0 || p->below > 2) return MCCE_EINVAL;
  const int64_t width = (int64_t)p->n * (1 + p->gated), wide = p->below == 2 ? 2ll * p->k : p->k, rows = p->n_layers * p->rows;
  if (saved && p->saved_dtype != p->dtype && p->saved_dtype != MCCE_E4M3) return MCCE_EINVAL;
  const bool bytes = saved && p->saved_dtype == MCCE_E4M3;
  if (!stride_ok(p->ld_y, width) || !stride_ok(p->ld_x, wide) || (add && !stride_ok(p->ld_add, p->k)) ||
      (saved && !stride_ok(p->ld_saved, wide)) || (h && !stride_ok(p->ld_h, p->k)))
    return MCCE_EINVAL;
  if ((w_up != nullptr) != (p->gated == 1) || (saved != nullptr) != (p->below > 0) || (scales != nullptr) != bytes) return MCCE_EINVAL;
  if (p->below ? add != nullptr : (h != nullptr || p->act != MCCE_ACT_NONE)) return MCCE_EINVAL;
  if (rows == 0) return MCCE_OK;
  if (!dout || !offsets || !w || !dx) return MCCE_EINVAL;
  const int e = elem(p->dtype), es = bytes ? 1 : e;
  if (!aligned(dout, e) || !aligned(offsets, 4) || !aligned(w, e) || !aligned(w_up, e) || !aligned(add, e) || !aligned(saved, es) ||
      !aligned(dx, e) || !aligned(h, e))
    return MCCE_EINVAL;
  Problem q = problem(*p, offsets);
  q.y = dout, q.w = w, q.w_up = w_up;
  q.ld_y = ld_or(p->ld_y, width);
  BackwardArgs& b = q.bwd;
  b.add = add, b.saved = saved, b.scales = (const uint8_t*)scales, b.dx = dx, b.h = h;
  b.ld_add = ld_or(p->ld_add, p->k), b.ld_saved = ld_or(p->ld_saved, wide), b.ld_dx = ld_or(p->ld_x, wide), b.ld_h = ld_or(p->ld_h, p->k);
  b.below = p->below, b.act = p->act, b.k = p->k, b.blocks = blocks_of(p->k);
  b.wide = wide_rows(add, b.ld_add, e) && wide_rows(saved, b.ld_saved, es) && wide_rows(dx, b.ld_dx, e) && wide_rows(h, b.ld_h, e);
  const Span sy = row_span(dout, rows, q.ld_y, width, e), soff = flat_span(offsets, (int64_t)p->n_layers * (p->n_experts + 1), 4);
  const Span sw = weight_span(*p, w, e), swu = weight_span(*p, w_up, e), sadd = row_span(add, rows, b.ld_add, p->k, e);
  const Span ssv = row_span(saved, rows, b.ld_saved, wide, es);
  const Span ssc = flat_span(scales, rows, (p->below == 2 ? 2 : 1) * (int64_t)b.blocks);
  const Span sdx = row_span(dx, rows, b.ld_dx, wide, e), sh = row_span(h, rows, b.ld_h, p->k, e);
  const size_t need = copies_for(kBackward, q, p->dtype).bytes(q.gated);
  if (need && (!workspace || !aligned(workspace, 16))) return MCCE_EINVAL;
  if (workspace_bytes < need) return MCCE_ENOSPC;
  const Span sws = flat_span(need ? workspace : nullptr, need);
  if (!apart(sws, {&sy, &soff, &sw, &swu, &sadd, &ssv, &ssc, &sdx, &sh}) || !same_or_apart(sdx, sadd) || !(bytes ? apart(sdx, {&ssv}) : same_or_apart(sdx, ssv)) || !apart(sdx, {&sy, &soff, &sw, &swu, &ssc, &sh}) ||
      !apart(sh, {&sy, &soff, &sw, &swu, &sadd, &ssv, &ssc}))
    return MCCE_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return code(run_product(kBackward, q, p->dtype, workspace, st));
}

extern "C" size_t mcce_expert_linear_workspace_bytes(const mcce_linear* p, const void* x, const void* w, const void* w_up) {
  if (!sizes_ok(p)) return 0;
  Problem q = problem(*p, nullptr);
  q.x = x, q.w = w, q.w_up = w_up, q.ld_x = ld_or(p->ld_x, p->k);
  return copies_for(kForward, q, p->dtype).bytes(q.gated);
}
extern "C" size_t mcce_expert_linear_backward_workspace_bytes(const mcce_linear* p, const void* dout, const void* w, const void* w_up) {
  if (!sizes_ok(p)) return 0;
  Problem q = problem(*p, nullptr);
  q.y = dout, q.w = w, q.w_up = w_up, q.ld_y = ld_or(p->ld_y, (int64_t)p->n * (1 + p->gated));
  return copies_for(kBackward, q, p->dtype).bytes(q.gated);
}
extern "C" size_t mcce_expert_linear_dweight_workspace_bytes(const mcce_linear* p, const void* dout, const void* x) {
  if (!sizes_ok(p)) return 0;
  return unpacked_bytes(*p) + bias_bytes(*p) + copies_for(kDweight, dweight_problem(*p, dout, x), p->dtype).bytes(p->gated);
}

extern "C" int mcce_expert_linear_dweight(const mcce_linear* p, const void* dout, const void* x, const void* scales,
                                          const int32_t* offsets, const void* add_dw, const void* add_dw_up, const void* add_db,
                                          const void* add_db_up, void* dw, void* dw_up, void* db, void* db_up, void* workspace,
                                          size_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(p)) return MCCE_EINVAL;
  const bool bytes = p->saved_dtype == MCCE_E4M3;
  if (!bytes && p->saved_dtype != p->dtype) return MCCE_EINVAL;
  const int64_t width = (int64_t)p->n * (1 + p->gated), rows = p->n_layers * p->rows;
  if (p->out_dtype != MCCE_F32 && p->out_dtype != p->dtype) return MCCE_EINVAL;
  if (!stride_ok(p->ld_y, width) || !stride_ok(p->ld_x, p->k)) return MCCE_EINVAL;
  if (!dw || !offsets || (dw_up != nullptr) != (p->gated == 1) || (db_up != nullptr) != (db != nullptr && p->gated) ||
      (scales != nullptr) != (bytes && rows > 0))
    return MCCE_EINVAL;
  if ((add_dw_up != nullptr) != (add_dw != nullptr && p->gated) || (add_db_up != nullptr) != (add_db != nullptr && p->gated) || (add_db && !db))
    return MCCE_EINVAL;
  if (rows && (!dout || !x)) return MCCE_EINVAL;
  const int e = elem(p->dtype), eo = elem(p->out_dtype), ex = bytes ? 1 : e;
  if (!aligned(dout, e) || !aligned(x, ex) || !aligned(offsets, 4) || !aligned(add_dw, eo) || !aligned(add_dw_up, eo) || !aligned(add_db, eo) ||
      !aligned(add_db_up, eo) || !aligned(dw, eo) || !aligned(dw_up, eo) || !aligned(db, eo) || !aligned(db_up, eo))
    return MCCE_EINVAL;
  const size_t need = mcce_expert_linear_dweight_workspace_bytes(p, dout, x);
  if (need && (!workspace || !aligned(workspace, 16))) return MCCE_EINVAL;
  if (workspace_bytes < need) return MCCE_ENOSPC;
  Problem q = problem(*p, offsets);
  const int64_t G = q.groups.G;
  q.y = dout, q.x = x, q.ld_y = ld_or(p->ld_y, width), q.ld_x = ld_or(p->ld_x, p->k);
  q.dw = dw, q.dw_up = dw_up, q.add_dw = add_dw, q.add_dw_up = add_dw_up, q.dw_f32 = p->out_dtype == MCCE_F32;
  auto dw_aligned = [&](int64_t bytes) {
    return aligned(dw, bytes) && aligned(dw_up, bytes) && aligned(add_dw, bytes) && aligned(add_dw_up, bytes) && q.ld_w * eo % bytes == 0 && q.step_w * eo % bytes == 0;
  };
  q.dw_wide = dw_aligned(16) ? 2 : dw_aligned(4 * eo) ? 1 : 0;
  const Span sy = row_span(dout, rows, q.ld_y, width, e), sx = row_span(x, rows, q.ld_x, p->k, ex);
  const Span ssc = flat_span(scales, rows, blocks_of(p->k)), soff = flat_span(offsets, (int64_t)p->n_layers * (p->n_experts + 1), 4);
  const Span saw = weight_span(*p, add_dw, eo), sawu = weight_span(*p, add_dw_up, eo), sab = flat_span(add_db, G * p->n, eo);
  const Span sabu = flat_span(add_db_up, G * p->n, eo), sdw = weight_span(*p, dw, eo), sdwu = weight_span(*p, dw_up, eo);
  const Span sdb = flat_span(db, G * p->n, eo), sdbu = flat_span(db_up, G * p->n, eo), sws = flat_span(need ? workspace : nullptr, need);
  if (!same_or_apart(sdw, saw) || !same_or_apart(sdwu, sawu) || !same_or_apart(sdb, sab) || !same_or_apart(sdbu, sabu) ||
      !apart(sdw, {&sy, &sx, &ssc, &soff, &sawu, &sab, &sabu, &sdwu, &sdb, &sdbu}) ||
      !apart(sdwu, {&sy, &sx, &ssc, &soff, &saw, &sab, &sabu, &sdb, &sdbu}) || !apart(sdb, {&sy, &sx, &ssc, &soff, &saw, &sawu, &sabu, &sdbu}) ||
      !apart(sdbu, {&sy, &sx, &ssc, &soff, &saw, &sawu, &sab}) ||
      !apart(sws, {&sy, &sx, &ssc, &soff, &saw, &sawu, &sab, &sabu, &sdw, &sdwu, &sdb, &sdbu}))
    return MCCE_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (bytes && rows) {
    const int64_t ld = (p->k + 7) & ~7ll;
    const cudaError_t err = run_unpack((const uint8_t*)x, (const uint8_t*)scales, p->dtype, rows, p->k, ld, q.ld_x, workspace, st);
    if (err != cudaSuccess) return MCCE_ECUDA;
    q.x = workspace, q.ld_x = ld;
  }
  const Problem given = q;   // the bias's gradient reads dout where it is
  cudaError_t err = run_product(kDweight, q, p->dtype, (uint8_t*)workspace + unpacked_bytes(*p) + bias_bytes(*p), st);
  if (err == cudaSuccess && db)
    err = run_bias_sums(given, p->dtype, add_db, add_db_up, db, db_up, (float*)((uint8_t*)workspace + unpacked_bytes(*p)), st);
  return code(err);
}

static bool checkpoint_ok(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, const void* q, const void* scales) {
  if (!plain_type(dtype) || rows < 0 || rows > 0x7fffffffll || d < 1 || d > MCCE_LINEAR_MAX_WIDTH || !stride_ok(ld_x, d) || !stride_ok(ld_q, d))
    return false;
  return rows == 0 || (x && q && scales && aligned(x, elem(dtype)));
}

extern "C" int mcce_checkpoint_pack(const void* x, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q, void* q, void* scales,
                                    void* cuda_stream) {
  if (!checkpoint_ok(x, dtype, rows, d, ld_x, ld_q, q, scales)) return MCCE_EINVAL;
  if (rows == 0) return MCCE_OK;
  const Span sx = row_span(x, rows, ld_or(ld_x, d), d, elem(dtype)), sq = row_span(q, rows, ld_or(ld_q, d), d, 1);
  const Span ssc = flat_span(scales, rows, blocks_of(d));
  if (!apart(sq, {&sx, &ssc}) || !apart(ssc, {&sx})) return MCCE_EINVAL;
  return code(run_pack(x, dtype, rows, d, ld_or(ld_x, d), ld_or(ld_q, d), (uint8_t*)q, (uint8_t*)scales, (cudaStream_t)cuda_stream));
}

extern "C" int mcce_checkpoint_unpack(const void* q, const void* scales, int32_t dtype, int64_t rows, int32_t d, int64_t ld_x, int64_t ld_q,
                                      void* x, void* cuda_stream) {
  if (!checkpoint_ok(x, dtype, rows, d, ld_x, ld_q, q, scales)) return MCCE_EINVAL;
  if (rows == 0) return MCCE_OK;
  const Span sx = row_span(x, rows, ld_or(ld_x, d), d, elem(dtype)), sq = row_span(q, rows, ld_or(ld_q, d), d, 1);
  const Span ssc = flat_span(scales, rows, blocks_of(d));
  if (!apart(sx, {&sq, &ssc})) return MCCE_EINVAL;
  return code(run_unpack((const uint8_t*)q, (const uint8_t*)scales, dtype, rows, d, ld_or(ld_x, d), ld_or(ld_q, d), x, (cudaStream_t)cuda_stream));
}
