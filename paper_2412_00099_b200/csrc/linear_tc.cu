// The experts' products on sorted rows on the 5th-generation tensor cores (bf16 rows and weights, fp32 sums).
//
// All three are products whose reduction lies along K-slabs of 64:
//   forward   D[feature, row] = sum_k w[feature, k] x[row, k]                  both operands with k along their rows
//   backward  D[feature, row] = sum_j w[j, feature] dout[row, j]               weights across their rows
//   dweight   D[j, feature]   = sum_r dout[r, j] x[r, feature]                 both across their rows; r runs over the group's rows
// Weight features are the 128 rows of the MMA and token rows its N dimension: groups of any size then cost what their rows rounded up to 16 cost,
// where 128-row tiles of tokens would waste a third of the work at 250 rows per expert.  A gated forward tile has 64 features: 32 gate rows, 32
// up rows and so on in turn, so that two neighbouring epilogue warps hold gate and up of the same features and swap half of their rows.
//
// One CTA per SM walks the tiles.  Warp 0 issues TMA loads into a ring of stages, warp 1 the MMAs into one of two TMEM buffers, eight warps
// bring the other buffer to memory, a feature per lane.  Every wait is bounded: when one gives up, the CTA notes it, lets its copies land, frees
// its TMEM and returns.
#include <cuda.h>

#include <type_traits>

#include "linear.cuh"
#include "tc_common.cuh"

namespace mcce {
namespace linear {

using namespace tc;

namespace {

__device__ uint32_t wait_error;   // set when a bounded wait gives up; read and cleared by mcce_expert_linear_status

constexpr int kTileM = 128;    // MMA rows
constexpr int kSlab = 64;      // reduction per stage: 64 bf16 = one 128-byte swizzled row
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr uint32_t kABytes = kTileM * kSlab * 2;
constexpr uint32_t kPanelBytes = kSlab * 128;   // an operand across its rows: 64 rows of 64 columns
constexpr int kBlockOfTiles = 16;   // row tiles of a group that are walked together, so that their rows stay in L2 for the next features

template <int KIND, bool GATED, int BN>
struct Cfg {
  static constexpr uint32_t kBBytes = BN * kSlab * 2;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  static constexpr uint32_t kSwapBytes = KIND == kForward && GATED ? 4 * 2 * 2 * 8 * 32 * 4 : 0;
  static constexpr uint32_t kCountBytes = KIND == kDweight ? 0 : ((MCCE_LINEAR_MAX_GROUPS + 1 + 33) * 4 + 127) & ~127;
  static constexpr uint32_t kFixed = 1024 + 512 + kSwapBytes + kCountBytes;
  static constexpr int kFit = (232448 - kFixed) / kStageBytes;
  static constexpr int kStages = kFit < 10 ? kFit : 10;
  static constexpr size_t kSmemBytes = kFixed + (size_t)kStages * kStageBytes;
  static constexpr int kRowBox = BN >= 64 ? 32 : 16;   // token rows per TMA copy
};

struct Maps {
  CUtensorMap a, a_up;   // weights; dweight: dout and its second half
  CUtensorMap b, b_up;   // rows; dweight: x
};

// Descriptor of an operand across its rows: panels of 64 columns (128 bytes), kPanelBytes apart; eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_across(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(kPanelBytes >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}

struct Item {
  int g, f0;        // group, first feature (dweight: first column of dout)
  int row, rows;    // first row among all, rows of the tile (dweight: the group's)
  int j0, half;     // dweight: first column of x; which half of dout
};

template <int KIND, bool GATED, int BN>
struct Walk {
  const Problem& p;
  const int* before;
  int64_t items;
  int FT, JT;   // tiles of features (dweight: of dout's columns), of x's columns
  __device__ __forceinline__ Walk(const Problem& p_, const int* before_) : p(p_), before(before_) {
    const int features = KIND == kBackward ? p.k : p.n, per = KIND == kForward && GATED ? kTileM / 2 : kTileM;
    FT = (features + per - 1) / per, JT = KIND == kDweight ? (p.k + BN - 1) / BN : 1;
    items = KIND == kDweight ? (int64_t)p.groups.G * (GATED ? 2 : 1) * FT * JT : (int64_t)before[p.groups.G] * FT;
  }
  __device__ __forceinline__ Item at(int64_t w) const {
    Item it;
    if (KIND == kDweight) {
      it.f0 = (int)(w % FT) * kTileM, w /= FT;
      it.j0 = (int)(w % JT) * BN, w /= JT;
      it.half = GATED ? (int)(w & 1) : 0;
      it.g = (int)(GATED ? w >> 1 : w);
      const GroupRows gr = group_rows(p.groups, it.g);
      it.row = (int)gr.first, it.rows = (int)gr.m;
    } else {
      it.g = find_group(before, p.groups.G, (int)(w / FT));
      const GroupRows gr = group_rows(p.groups, it.g);
      const int tiles = before[it.g + 1] - before[it.g];
      const int64_t in = w - (int64_t)before[it.g] * FT;
      const int block = (int)(in / (kBlockOfTiles * FT)), rest = (int)(in % (kBlockOfTiles * FT));
      const int wide = min(kBlockOfTiles, tiles - block * kBlockOfTiles);
      const int tile = block * kBlockOfTiles + rest % wide;
      it.f0 = rest / wide * (GATED && KIND == kForward ? kTileM / 2 : kTileM);
      const int m = (int)gr.m, each = ((m + tiles - 1) / tiles + 15) & ~15;   // tiles of equal size; none is empty
      it.row = (int)gr.first + tile * each, it.rows = min(each, m - tile * each);
      it.j0 = it.half = 0;
    }
    return it;
  }
  __device__ __forceinline__ int slabs(const Item& it) const {
    if (KIND == kDweight) return (it.rows + kSlab - 1) / kSlab;
    return KIND == kForward ? (p.k + kSlab - 1) / kSlab : (GATED ? 2 : 1) * ((p.n + kSlab - 1) / kSlab);
  }
};

template <int KIND, bool GATED, int BN>
__global__ void __launch_bounds__(kThreads, 1) linear_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Problem p) {
  using C = Cfg<KIND, GATED, BN>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_al = smem_raw + (smem_base - smem_u32(smem_raw));
  uint8_t* rest = smem_al + (size_t)C::kStages * C::kStageBytes;
  float* swap = (float*)rest;   // [pair of warps][buffer][direction][8 rows][32 lanes]
  int* before = (int*)(rest + C::kSwapBytes);
  uint64_t* bars = (uint64_t*)(rest + C::kSwapBytes + C::kCountBytes);
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * C::kStages;
  const uint32_t bar_tfull = bar_empty + 8 * C::kStages, bar_tempty = bar_tfull + 16, bar_swap = bar_tempty + 16;
  uint32_t* tmem_slot = (uint32_t*)(bars + 2 * C::kStages + 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar_tfull + 8 * b, 1);
      mbar_init(bar_tempty + 8 * b, kEpilogueWarps);
    }
    for (int b = 0; b < 4; ++b) mbar_init(bar_swap + 8 * b, 2);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 2 * BN);
  if (KIND != kDweight) count_tiles(p.groups, BN, before, before + p.groups.G + 1);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const Walk<KIND, GATED, BN> walk(p, before);

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool alive = true;
      for (int64_t w = blockIdx.x; w < walk.items && alive; w += gridDim.x) {
        const Item it = walk.at(w);
        const int slabs = walk.slabs(it), part = GATED && KIND == kBackward ? slabs / 2 : slabs;
        const int panels = KIND == kDweight ? min(BN / 64, (p.k - it.j0 + 63) / 64) : 0;
        const int boxes = (it.rows + C::kRowBox - 1) / C::kRowBox;
        const uint32_t tx = kABytes + (KIND == kDweight ? panels * kPanelBytes : (uint32_t)boxes * C::kRowBox * kSlab * 2);
        for (int kt = 0; kt < slabs; ++kt) {
          if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, &wait_error, 1u)) {
            alive = false;
            break;
          }
          const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kABytes, full = bar_full + 8 * stage;
          mbar_expect_tx(full, tx);
          if (KIND == kForward) {
            const int x = kt * kSlab;
            if (GATED) {
#pragma unroll
              for (int i = 0; i < 4; ++i) tma_load_3d(sa + i * 4096, i & 1 ? &maps.a_up : &maps.a, x, it.f0 + (i >> 1) * 32, it.g, full);
            } else {
              tma_load_3d(sa, &maps.a, x, it.f0, it.g, full);
            }
            for (int i = 0; i < boxes; ++i) tma_load_2d(sb + i * C::kRowBox * 128, &maps.b, x, it.row + i * C::kRowBox, full);
          } else if (KIND == kBackward) {
            const bool up = kt >= part;
            const int x = (up ? kt - part : kt) * kSlab;
            tma_load_3d(sa, up ? &maps.a_up : &maps.a, it.f0, x, it.g, full);
            tma_load_3d(sa + kPanelBytes, up ? &maps.a_up : &maps.a, it.f0 + 64, x, it.g, full);
            for (int i = 0; i < boxes; ++i) tma_load_2d(sb + i * C::kRowBox * 128, up ? &maps.b_up : &maps.b, x, it.row + i * C::kRowBox, full);
          } else {
            const int y = it.row + kt * kSlab;
            tma_load_2d(sa, it.half ? &maps.a_up : &maps.a, it.f0, y, full);
            tma_load_2d(sa + kPanelBytes, it.half ? &maps.a_up : &maps.a, it.f0 + 64, y, full);
            for (int i = 0; i < panels; ++i) tma_load_2d(sb + i * kPanelBytes, &maps.b, it.j0 + 64 * i, y, full);
          }
          if (++stage == C::kStages) stage = 0, phase ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    // The whole warp walks along: in dweight's last slab its lanes clear the rows that belong to the next group.
    uint32_t stage = 0, phase = 0, acc = 0;
    bool alive = true;
    for (int64_t w = blockIdx.x; w < walk.items && alive; w += gridDim.x) {
      const Item it = walk.at(w);
      const int slabs = walk.slabs(it);
      if (slabs == 0) continue;
      const int cols = KIND == kDweight ? min(BN, p.k - it.j0) : it.rows;
      // fp32 sums of bf16, M = 128, N; a set bit 15 / 16: A / B lies across its rows
      const uint32_t idesc = instr_desc((uint32_t)(cols + 15) & ~15u) | (KIND != kForward ? 1u << 15 : 0u) | (KIND == kDweight ? 1u << 16 : 0u);
      const uint32_t buf = acc & 1u;
      if (!mbar_wait(bar_tempty + 8 * buf, ((acc >> 1) & 1u) ^ 1u, abort_flag, &wait_error, 2u)) break;
      ++acc;
      tc_fence_after();
      const uint32_t d = tmem_base + buf * BN;
      for (int kt = 0; kt < slabs; ++kt) {
        if (!mbar_wait(bar_full + 8 * stage, phase, abort_flag, &wait_error, 3u)) {
          alive = false;
          break;
        }
        const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kABytes;
        int steps = kSlab / 16;
        if (KIND == kDweight && it.rows - kt * kSlab < kSlab) {
          const int valid = it.rows - kt * kSlab;
          steps = (valid + 15) / 16;
          // both operands: zero times a NaN of the next group would not be zero
          const int n16 = (steps * 16 - valid) * 8, panels = 2 + (cols + 63) / 64;
          for (int i = lane; i < n16 * panels; i += 32)
            *(uint4*)(smem_al + (size_t)stage * C::kStageBytes + (size_t)(i / n16) * kPanelBytes + valid * 128 + (i % n16) * 16) =
                make_uint4(0u, 0u, 0u, 0u);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        tc_fence_after();
        if (lane == 0) {
          for (int k = 0; k < steps; ++k) {
            const uint64_t ad = KIND == kForward ? smem_desc(sa + k * 32) : smem_desc_across(sa + k * 2048);
            const uint64_t bd = KIND == kDweight ? smem_desc_across(sb + k * 2048) : smem_desc(sb + k * 32);
            umma_bf16(d, ad, bd, idesc, (kt | k) != 0 ? 1u : 0u);
          }
          umma_commit(bar_empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == C::kStages) stage = 0, phase ^= 1u;
      }
      if (alive && lane == 0) umma_commit(bar_tfull + 8 * buf);
      __syncwarp();
    }
  } else {
    const int quad = warp & 3, team = (warp - 2) >> 2;   // TMEM lanes this warp may read; which half of the chunks it takes
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    uint32_t acc = 0, swaps = 0;
    bool alive = true;
    for (int64_t w = blockIdx.x; w < walk.items && alive; w += gridDim.x) {
      const Item it = walk.at(w);
      const bool sums = walk.slabs(it) > 0;
      const uint32_t buf = acc & 1u;
      if (sums) {
        if (!mbar_wait(bar_tfull + 8 * buf, (acc >> 1) & 1u, abort_flag, &wait_error, 4u)) break;
        ++acc;
        tc_fence_after();
      }
      const uint32_t t0 = tmem_base + lane_addr + buf * BN;
      if constexpr (KIND == kDweight) {
        const int cols = min(BN, p.k - it.j0), i = it.f0 + quad * 32 + lane;
        const void* add = it.half ? p.add_dw_up : p.add_dw;
        void* dw = it.half ? p.dw_up : p.dw;
        const int64_t at = it.g * p.step_w + (int64_t)i * p.ld_w + it.j0;
        const bool on = i < p.n;
        for (int c = 16 * team; c < cols; c += 32) {
          float v[16] = {};
          __syncwarp();   // the loads from TMEM take the whole warp
          if (sums) {
            tmem_ld16(t0 + c, v);
            tmem_ld_wait();
          }
          if (!on) continue;
          const int left = min(16, cols - c);
          if (p.dw_f32) {
            float* o = (float*)dw + at + c;
            const float* a = add ? (const float*)add + at + c : nullptr;
            if (p.dw_wide && left == 16) {
#pragma unroll
              for (int j = 0; j < 16; j += 4) {
                float4 q = a ? *(const float4*)(a + j) : make_float4(0.f, 0.f, 0.f, 0.f);
                q.x += v[j], q.y += v[j + 1], q.z += v[j + 2], q.w += v[j + 3];
                *(float4*)(o + j) = q;
              }
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < left) o[j] = v[j] + (a ? a[j] : 0.f);
            }
          } else {
            __nv_bfloat16* o = (__nv_bfloat16*)dw + at + c;
            const __nv_bfloat16* a = add ? (const __nv_bfloat16*)add + at + c : nullptr;
            if (p.dw_wide && left == 16) {
#pragma unroll
              for (int j = 0; j < 16; j += 8) {
                uint4 q = a ? *(const uint4*)(a + j) : make_uint4(0u, 0u, 0u, 0u);
                __nv_bfloat162* h = (__nv_bfloat162*)&q;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const float2 f = __bfloat1622float2(h[u]);
                  h[u] = __floats2bfloat162_rn(f.x + v[j + 2 * u], f.y + v[j + 2 * u + 1]);
                }
                *(uint4*)(o + j) = q;
              }
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < left) store_as(o + j, v[j] + (a ? load_as_float(a + j) : 0.f));
            }
          }
        }
      } else if constexpr (KIND == kForward && GATED) {
        // even quadrants hold z, odd ones z_up of the same 32 features; of every 16 rows the first 8 are finished by the even warp
        const int pair = (quad >> 1) * 2 + team, up = quad & 1;
        const Forward<__nv_bfloat16, true> e(p.fwd, it.g, it.f0 + (quad >> 1) * 32 + lane);
        for (int c = 16 * team; c < it.rows && alive; c += 32, ++swaps) {
          float v[16];
          __syncwarp();
          tmem_ld16(t0 + c, v);
          tmem_ld_wait();
          float* mine = swap + (pair * 2 + (swaps & 1)) * 512 + up * 256;
          const float* theirs = swap + (pair * 2 + (swaps & 1)) * 512 + (up ^ 1) * 256;
#pragma unroll
          for (int j = 0; j < 8; ++j) mine[j * 32 + lane] = up ? v[j] : v[8 + j];
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_swap + 8 * pair);
          if (!mbar_wait(bar_swap + 8 * pair, swaps & 1u, abort_flag, &wait_error, 5u)) {
            alive = false;
            break;
          }
          const int64_t row = it.row + c + up * 8;
          const int left = it.rows - c - up * 8;
          typename Forward<__nv_bfloat16, true>::Pre pre[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < left) pre[j] = e.load(row + j);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float other = theirs[j * 32 + lane];
            if (j < left) e.store(row + j, up ? other : v[j], up ? v[8 + j] : other, pre[j]);
          }
        }
      } else {
        typedef typename std::conditional<KIND == kForward, Forward<__nv_bfloat16, false>, Backward<__nv_bfloat16>>::type Epilogue;
        const int f = it.f0 + quad * 32 + lane;
        const Epilogue e = [&] {
          if constexpr (KIND == kForward) return Epilogue(p.fwd, it.g, f);
          else return Epilogue(p.bwd, it.g, f);
        }();
        for (int c = 16 * team; c < it.rows; c += 32) {
          const int64_t row = it.row + c;
          const int left = it.rows - c;
          typename Epilogue::Pre pre[16];
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j < left) pre[j] = e.load(row + j);
          float v[16];
          __syncwarp();
          tmem_ld16(t0 + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j < left) e.store(row + j, v[j], 0.f, pre[j]);
        }
      }
      if (sums) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_tempty + 8 * buf);
      }
    }
  }

  __syncwarp();
  if (*abort_flag) {
    // copies and MMAs still in flight land before shared memory and TMEM are released
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem_base, 2 * BN);
}

// ---- host ---------------------------------------------------------------------------------------------------------
bool encode(CUtensorMap* m, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t one[3] = {1, 1, 1};
  EncodeFn fn = encode_fn();
  return fn && fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [rows, cols], a box of 64 columns
bool map_rows(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {kSlab, (cuuint32_t)box_rows};
  return encode(m, base, 2, dims, strides, box);
}
// [groups, n, k]: what lies outside a matrix is filled with zeros, not with the next matrix
bool map_weights(CUtensorMap* m, const void* base, const Problem& p, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)p.k, (cuuint64_t)p.n, (cuuint64_t)p.groups.G};
  const cuuint64_t strides[2] = {(cuuint64_t)p.ld_w * 2, (cuuint64_t)(p.groups.G > 1 ? p.step_w : (p.n * p.ld_w + 7) & ~7ll) * 2};
  const cuuint32_t box[3] = {kSlab, (cuuint32_t)box_rows, 1};
  return encode(m, base, 3, dims, strides, box);
}

template <int KIND, bool GATED, int BN>
cudaError_t launch(const Problem& p, cudaStream_t st) {
  using C = Cfg<KIND, GATED, BN>;
  static int cache[64] = {0};
  int sms = 0;
  const cudaError_t e = sm_count_and_smem_optin(linear_tc_kernel<KIND, GATED, BN>, C::kSmemBytes, cache, &sms);
  if (e != cudaSuccess) return e;
  Maps m;
  bool ok;
  const int64_t rows = p.L * p.groups.R;
  const int kind_features = KIND == kBackward ? p.k : p.n, per = KIND == kForward && GATED ? kTileM / 2 : kTileM;
  const int64_t FT = (kind_features + per - 1) / per;
  int64_t most;
  if (KIND == kDweight) {
    const __nv_bfloat16* y = (const __nv_bfloat16*)p.y;
    ok = map_rows(&m.a, y, rows, p.n, p.ld_y, kSlab) && map_rows(&m.b, p.x, rows, p.k, p.ld_x, kSlab) &&
         (!GATED || map_rows(&m.a_up, y + p.n, rows, p.n, p.ld_y, kSlab));
    most = (int64_t)p.groups.G * (GATED ? 2 : 1) * FT * ((p.k + BN - 1) / BN);
  } else if (KIND == kForward) {
    const int box = GATED ? 32 : kTileM;
    ok = map_weights(&m.a, p.w, p, box) && (!GATED || map_weights(&m.a_up, p.w_up, p, box)) && map_rows(&m.b, p.x, rows, p.k, p.ld_x, C::kRowBox);
    most = (rows / BN + p.groups.G) * FT;
  } else {
    const __nv_bfloat16* y = (const __nv_bfloat16*)p.y;
    ok = map_weights(&m.a, p.w, p, kSlab) && (!GATED || map_weights(&m.a_up, p.w_up, p, kSlab)) &&
         map_rows(&m.b, y, rows, p.n, p.ld_y, C::kRowBox) && (!GATED || map_rows(&m.b_up, y + p.n, rows, p.n, p.ld_y, C::kRowBox));
    most = (rows / BN + p.groups.G) * FT;
  }
  if (!ok) return cudaErrorInvalidValue;
  linear_tc_kernel<KIND, GATED, BN><<<(unsigned)(most < sms ? most : sms), kThreads, C::kSmemBytes, st>>>(m, p);
  return cudaGetLastError();
}

template <int KIND, bool GATED>
cudaError_t launch_rows(const Problem& p, cudaStream_t st) {
  const int64_t each = p.L * p.groups.R / p.groups.G;
  if (each <= 24) return launch<KIND, GATED, 32>(p, st);
  if (each <= 96) return launch<KIND, GATED, 128>(p, st);
  return launch<KIND, GATED, 256>(p, st);
}

bool tma_rows(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

}  // namespace

bool tensor_applicable(Kind kind, const Problem& p, int32_t dtype) {
  if (dtype != MCCE_BF16) return false;
  if (kind == kDweight) return p.L * p.groups.R > 0 && tma_rows(p.y, p.ld_y) && tma_rows(p.x, p.ld_x) && (!p.gated || p.n % 8 == 0);
  if (!tma_rows(p.w, p.ld_w) || !tma_rows(p.w_up, p.ld_w) || (p.groups.G > 1 && p.step_w % 8)) return false;
  if (kind == kForward) return tma_rows(p.x, p.ld_x);
  return tma_rows(p.y, p.ld_y) && (!p.gated || p.n % 8 == 0);
}

cudaError_t run_tensor(Kind kind, const Problem& p, cudaStream_t st) {
  if (kind == kForward) return p.gated ? launch_rows<kForward, true>(p, st) : launch_rows<kForward, false>(p, st);
  if (kind == kBackward) return p.gated ? launch_rows<kBackward, true>(p, st) : launch_rows<kBackward, false>(p, st);
  return p.gated ? launch<kDweight, true, 256>(p, st) : launch<kDweight, false, 256>(p, st);
}

}  // namespace linear
}  // namespace mcce

extern "C" int mcce_expert_linear_status(void* cuda_stream) {
  cudaStream_t st = (cudaStream_t)cuda_stream;
  uint32_t word = 0;
  const uint32_t none = 0;
  if (cudaMemcpyFromSymbolAsync(&word, mcce::linear::wait_error, 4, 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess)
    return MCCE_ECUDA;
  if (!word) return MCCE_OK;
  if (cudaMemcpyToSymbolAsync(mcce::linear::wait_error, &none, 4, 0, cudaMemcpyHostToDevice, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess)
    return MCCE_ECUDA;
  return MCCE_ETIMEOUT;
}
