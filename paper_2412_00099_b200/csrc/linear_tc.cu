// The experts' products on sorted rows on the 5th-generation tensor cores (bf16 rows and weights, fp32 sums).
//
// All three are products whose reduction lies along slabs of 64 (dweight: 128):
//   forward   D[feature, row] = sum_k w[feature, k] x[row, k]                  both operands with k along their rows
//   backward  D[feature, row] = sum_j w[j, feature] dout[row, j]               weights across their rows
//   dweight   D[j, feature]   = sum_r dout[r, j] x[r, feature]                 both across their rows; r runs over the group's rows
// Weight features are the 128 rows of the MMA and token rows its N dimension: groups of any size then cost what their rows rounded up to 16 cost,
// where 128-row tiles of tokens would waste a third of the work at 250 rows per expert.  A gated forward tile has 64 features: 64
// gate rows, then 64 up rows, so that two epilogue warps hold gate and up of the same features and swap half of their rows.
//
// One CTA per SM, or a pair on two, walks the tiles.  Warp 0 issues TMA loads into a ring of stages, warp 1 the MMAs into one of two TMEM buffers, 8 or 16
// warps bring the other buffer to memory: from a feature per lane, as TMEM gives it, through shared memory to eight columns of a row per lane.
// Every wait is bounded: when one gives up, the CTA notes it, lets its copies land, frees its TMEM and returns.
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
constexpr int kSwapStride = 36;   // floats of a row: reading eight columns per lane, four lanes a row, then meets every bank once
constexpr int kBlockOfTiles = 8;  // row tiles of a group that are walked together, so that their rows stay in L2 for the next features

// How CTAs of a cluster work together: each for itself; a pair on one tile; several on parts of one tile's reduction.
enum Share { kAlone = 0, kPair = 1, kSplit = 2 };
constexpr int most_parts(int bn) { return bn <= 64 ? 4 : 2; }   // CTAs on one reduction: what rank 0 has room for

template <int KIND, bool GATED, int BN, int SHARE>
struct Cfg {
  static constexpr bool PAIR = SHARE == kPair;
  static constexpr int kCtas = PAIR ? 2 : 1;
  static constexpr int kFeatures = kTileM * kCtas / (KIND == kForward && GATED ? 2 : 1);   // of a tile
  // Reduction per stage.  Along an operand's rows 64 bf16 are a swizzled row of 128 bytes; dweight's operands lie across their rows, and the fewer copies of
  // 128 rows win (8192 x 4096 x 4096: 197 us, with 64 rows 203).
  static constexpr int kSlab = KIND == kDweight ? 128 : 64;
  static constexpr uint32_t kABytes = kTileM * kSlab * 2;
  static constexpr uint32_t kBBytes = BN / kCtas * kSlab * 2;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  // Epilogue warps, four teams (a gated layer and dweight: two) of a warp per TMEM quadrant.  They have few instructions that do not wait for another:
  // 16 of them take a gated layer's gradient through in 2/3 of the time of 8.
  static constexpr int kTeams = KIND == kDweight || (KIND == kForward && GATED) ? 2 : 4;
  static constexpr int kEpilogueWarps = 4 * kTeams, kClearWarp = 2 + kEpilogueWarps;
  // Sums of 8 (gated: 16) rows x 32 features per epilogue warp, on their way from a feature per lane to a row per four lanes; gated: two buffers;
  // dweight: 32 x 32.
  static constexpr uint32_t kSwapBytes =
      kEpilogueWarps * (KIND == kDweight ? 4096 : 8 * kSwapStride * 4 * (KIND == kForward && GATED ? 4 : 1));
  static constexpr uint32_t kCountBytes = KIND == kDweight ? 0 : ((MCCE_LINEAR_MAX_GROUPS + 1 + 33) * 4 + 127) & ~127;
  static constexpr uint32_t kPartBytes = SHARE == kSplit ? (most_parts(BN) - 1) * BN * kTileM * 4 : 0;   // the other CTAs' sums, in rank 0's
  static constexpr uint32_t kFixed = 1024 + 512 + kSwapBytes + kCountBytes + kPartBytes;
  static constexpr int kFit = (232448 - kFixed) / kStageBytes;
  static constexpr int kStages = kFit < 10 ? kFit : 10;
  static constexpr int kThreads = 32 * (2 + kEpilogueWarps + (KIND == kDweight ? 1 : 0));
  static constexpr size_t kSmemBytes = kFixed + (size_t)kStages * kStageBytes;
  static constexpr int kRowBox = BN / kCtas;   // most rows per TMA copy
};

struct Maps {
  CUtensorMap a[2], a_up[2];   // weights; dweight: dout and its second half, 128 and 64 rows at a time
  CUtensorMap b[4], b_up[4];   // rows, boxes of 1/4, 2/4, 3/4 and 4/4 of a CTA's most; dweight: x, 128 and 64 rows at a time
  CUtensorMap d, d_up;    // dweight: dw, where it is written by copies
  int d_copies;
  int a_whole, b_whole;   // operands across their rows: one copy brings both panels of 64 columns; forward: all matrices in one map of their rows
  int a_step;             // forward, then: rows from one matrix to the next
};

// Descriptor of an operand across its rows: panels of 64 columns (128 bytes), `panel` bytes apart; eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_across(uint32_t addr, uint32_t panel) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(panel >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// 8 and 32 consecutive fp32 columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
      "%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// TMA copies into this CTA's shared memory; in a pair the barrier may be the other CTA's.
#define MCCE_TMA_LOAD(DIMS, COORDS, ...)                                                                                              \
  if (PAIR)                                                                                                                           \
    asm volatile("cp.async.bulk.tensor." DIMS                                                                                         \
                 ".cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {" COORDS "}], [%2];" ::"r"(dst),      \
                 "l"(map), "r"(bar), __VA_ARGS__                                                                                      \
                 : "memory");                                                                                                         \
  else                                                                                                                                \
    asm volatile("cp.async.bulk.tensor." DIMS ".shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {" COORDS "}], [%2];"  \
                 ::"r"(dst),                                                                                                          \
                 "l"(map), "r"(bar), __VA_ARGS__                                                                                      \
                 : "memory")
template <bool PAIR>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  MCCE_TMA_LOAD("2d", "%3, %4", "r"(x), "r"(y));
}
template <bool PAIR>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  MCCE_TMA_LOAD("3d", "%3, %4, %5", "r"(x), "r"(y), "r"(z));
}
template <bool PAIR>
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int u, uint32_t bar) {
  MCCE_TMA_LOAD("4d", "%3, %4, %5, %6", "r"(x), "r"(y), "r"(z), "r"(u));
}
#undef MCCE_TMA_LOAD
// `count` panels of 64 columns from column x, `panel` bytes each, rows from y on, of matrix g.  The map's dimensions: column in a panel, row, (panel,) matrix.
template <bool PAIR>
__device__ __forceinline__ void load_panels(uint32_t dst, const CUtensorMap* map, bool whole, int count, uint32_t panel, int x, int y, int g,
                                            uint32_t bar) {
  if (whole) load_4d<PAIR>(dst, map, 0, y, x / 64, g, bar);
  else
    for (int i = 0; i < count; ++i) load_3d<PAIR>(dst + i * panel, map, x + 64 * i, y, g, bar);
}

// ---- pairs of CTAs: the even one (rank 0) leads, its barriers say when both CTAs' operands have landed ----------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t leaders(uint32_t addr) {   // the same place in rank 0's shared memory
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// mbar_wait by a whole warp, with one answer: lanes that went on while another gives up would wait for it without a limit
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* err, uint32_t code,
                                          unsigned long long limit_ns = kWaitLimitNs) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, err, code, limit_ns));
}
// The same for what other CTAs of the cluster wrote
__device__ __forceinline__ bool warp_wait_cluster(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* err, uint32_t code,
                                                  unsigned long long limit_ns) {
  const bool ok = warp_wait(bar, parity, abort_flag, err, code, limit_ns);
  asm volatile("fence.acq_rel.cluster;" ::: "memory");
  return ok;
}
// Without ordering what this thread did before: a release at cluster scope waits for all of its stores.
__device__ __forceinline__ void arrive_at_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else umma_bf16(d, a, b, idesc, accumulate);
}
// Arrives, in both CTAs of a pair, once every MMA issued so far has completed.
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
  else umma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void take_tmem(uint32_t slot, uint32_t cols) {
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tmem_alloc(slot, cols);
  }
}
template <bool PAIR>
__device__ __forceinline__ void free_tmem(uint32_t addr, uint32_t cols) {
  if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
  else tmem_dealloc(addr, cols);
}

// 32 rows x 32 columns of sums, a row per lane, brought to memory (added to what is there) with four columns per lane, a row per eight lanes: whole
// sectors of 64 (bf16) or 128 neighbouring bytes, where a row per lane wrote 32 rows with every instruction.  They turn in shared memory, 16 bytes
// at a time, a row's units rotated by its number so that neither side meets a bank twice.
template <typename O>
__device__ __forceinline__ void store_block(uint8_t* buffer, const float (&v)[32], O* o, const O* add, int64_t ld, int rows, int cols, bool wide) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *(float4*)(buffer + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  __syncwarp();
  const int unit = lane & 7, count = min(4, cols - 4 * unit), r0 = lane >> 3;
  if (count <= 0) return;
  if (!wide || count < 4) {
    for (int r = r0; r < min(32, rows); r += 4)
      for (int j = 0; j < count; ++j)
        store_as(o + r * ld + 4 * unit + j, ((const float*)(buffer + r * 128 + ((unit ^ (r & 7)) << 4)))[j] +
                                                (add ? load_as_float(add + r * ld + 4 * unit + j) : 0.f));
    return;
  }
  float4 x[8];
  typedef typename std::conditional<sizeof(O) == 4, float4, uint2>::type Four;
  Four a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = Four{};
    if (add) a[i] = *(const Four*)(add + min(r0 + 4 * i, rows - 1) * ld + 4 * unit);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = *(const float4*)(buffer + (r0 + 4 * i) * 128 + ((unit ^ ((r0 + 4 * i) & 7)) << 4));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    O* to = o + (r0 + 4 * i) * ld + 4 * unit;
    Four v;
    if constexpr (sizeof(O) == 4) {
      v = make_float4(x[i].x + a[i].x, x[i].y + a[i].y, x[i].z + a[i].z, x[i].w + a[i].w);
    } else {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(x[i].x + __uint_as_float(a[i].x << 16), x[i].y + __uint_as_float(a[i].x & 0xffff0000u));
      const __nv_bfloat162 hi = __floats2bfloat162_rn(x[i].z + __uint_as_float(a[i].y << 16), x[i].w + __uint_as_float(a[i].y & 0xffff0000u));
      v = make_uint2(*(const uint32_t*)&lo, *(const uint32_t*)&hi);
    }
    if (r0 + 4 * i < rows) *(Four*)to = v;
  }
}

// This lane's eight columns of its row among eight
__device__ __forceinline__ void row_of(const float* buffer, int first, float (&v)[8]) {
  const int lane = threadIdx.x & 31;
  const float4* p = (const float4*)(buffer + (first + (lane >> 2)) * kSwapStride + 8 * (lane & 3));
  const float4 a = p[0], b = p[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

struct Item {
  int g, f0;        // group, first feature (dweight: first column of dout)
  int row, rows;    // first row among all, rows of the tile (dweight: the group's)
  int j0, half;     // dweight: first column of x; which half of dout
};

template <int KIND, bool GATED, int BN, int SHARE>
struct Walk {
  static constexpr int kFeatures = Cfg<KIND, GATED, BN, SHARE>::kFeatures;
  const Problem& p;
  const int* before;
  int first, step, items;   // this CTA's (cluster's) tiles: first, first + step ..
  int FT, JT;   // tiles of features (dweight: of dout's columns), of x's columns
  __device__ __forceinline__ Walk(const Problem& p_, const int* before_) : p(p_), before(before_) {
    const int features = KIND == kBackward ? p.k : p.n;
    const int ctas = SHARE == kAlone ? 1 : cluster_size();
    first = blockIdx.x / ctas, step = gridDim.x / ctas;
    FT = (features + kFeatures - 1) / kFeatures, JT = KIND == kDweight ? (p.k + BN - 1) / BN : 1;
    items = KIND == kDweight ? p.groups.G * (GATED ? 2 : 1) * FT * JT : before[p.groups.G] * FT;   // fits: the launch sees to it
    // A cluster with one reduction takes one tile, and there are as many clusters as tiles; more tiles can only be rows that descending offsets name twice.
    if (SHARE == kSplit) items = min(items, step);
  }
  __device__ __forceinline__ Item decode(int w) const {
    Item it;
    if (KIND == kDweight) {
      it.f0 = w % FT * kFeatures, w /= FT;
      it.j0 = w % JT * BN, w /= JT;
      it.half = GATED ? w & 1 : 0;
      it.g = GATED ? w >> 1 : w;
      const GroupRows gr = group_rows(p.groups, it.g);
      it.row = (int)gr.first, it.rows = (int)gr.m;
    } else {
      it.g = find_group(before, p.groups.G, w / FT);
      const GroupRows gr = group_rows(p.groups, it.g);
      const int tiles = before[it.g + 1] - before[it.g];
      const int in = w - before[it.g] * FT;
      const int block = in / (kBlockOfTiles * FT), rest = in % (kBlockOfTiles * FT);
      const int wide = min(kBlockOfTiles, tiles - block * kBlockOfTiles);
      const int tile = block * kBlockOfTiles + rest % wide;
      it.f0 = rest / wide * kFeatures;
      const int m = (int)gr.m, each = ((m + tiles - 1) / tiles + 15) & ~15;   // tiles of equal size; none is empty
      it.row = (int)gr.first + tile * each, it.rows = min(each, m - tile * each);
      it.j0 = it.half = 0;
    }
    return it;
  }
  // The i-th tile, by a whole warp: its lanes work out 32 tiles at a time (divisions and loads of offsets are paid once for them), `mine` is
  // the lane's.  False behind the last one.
  __device__ __forceinline__ bool at(int i, Item& mine, Item& it) const {
    const int64_t w = first + (int64_t)i * step;
    if (w >= items) return false;
    const int lane = threadIdx.x & 31;
    if ((i & 31) == 0) {
      const int64_t own = w + (int64_t)lane * step;
      mine = decode(own < items ? (int)own : items - 1);
    }
    const int from = i & 31;
    it.g = __shfl_sync(0xffffffffu, mine.g, from), it.f0 = __shfl_sync(0xffffffffu, mine.f0, from);
    it.row = __shfl_sync(0xffffffffu, mine.row, from), it.rows = __shfl_sync(0xffffffffu, mine.rows, from);
    it.j0 = KIND == kDweight ? __shfl_sync(0xffffffffu, mine.j0, from) : 0;
    it.half = KIND == kDweight && GATED ? __shfl_sync(0xffffffffu, mine.half, from) : 0;
    return true;
  }
  // N of the tile's MMAs: its rows; its columns of x, in whole panels for each CTA
  __device__ __forceinline__ int wide(const Item& it) const {
    if (KIND == kDweight) return (min(BN, p.k - it.j0) + 64 * Cfg<KIND, GATED, BN, SHARE>::kCtas - 1) & ~(64 * Cfg<KIND, GATED, BN, SHARE>::kCtas - 1);
    return (it.rows + 15) & ~15;
  }
  // The slabs of a tile that this CTA multiplies: all, or (several CTAs on its reduction) its share of them
  __device__ __forceinline__ void range(const Item& it, int place, int& from, int& to) const {
    from = 0, to = slabs(it);
    if (SHARE != kSplit) return;
    const int each = (to + (int)cluster_size() - 1) / (int)cluster_size();
    from = min(place * each, to), to = min(from + each, to);
  }
  __device__ __forceinline__ int slabs(const Item& it) const {
    constexpr int kSlab = Cfg<KIND, GATED, BN, SHARE>::kSlab;
    if (KIND == kDweight) return (it.rows + kSlab - 1) / kSlab;
    return KIND == kForward ? (p.k + kSlab - 1) / kSlab : (GATED ? 2 : 1) * ((p.n + kSlab - 1) / kSlab);
  }
};

// One CTA, or a pair of CTAs that share a tile: each has half of its features (128 MMA rows, accumulated in its own TMEM) and half of its
// rows (dweight: of x's columns) in shared memory, and the leader's MMAs read both halves.  A pair takes in a third less than two single CTAs for
// the same products.
template <int KIND, bool GATED, int BN, int SHARE>
__global__ void __launch_bounds__(Cfg<KIND, GATED, BN, SHARE>::kThreads, 1) linear_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Problem p) {
  using C = Cfg<KIND, GATED, BN, SHARE>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_al = smem_raw + (smem_base - smem_u32(smem_raw));
  uint8_t* rest = smem_al + (size_t)C::kStages * C::kStageBytes;
  float* swap = (float*)rest;
  int* before = (int*)(rest + C::kSwapBytes);
  uint64_t* bars = (uint64_t*)(rest + C::kSwapBytes + C::kCountBytes);
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * C::kStages;
  const uint32_t bar_tfull = bar_empty + 8 * C::kStages, bar_tempty = bar_tfull + 16, bar_swap = bar_tempty + 16, bar_tail = bar_swap + 32;
  const uint32_t bar_parts = bar_tail + 8 * C::kStages;
  uint32_t* tmem_slot = (uint32_t*)(bars + 3 * C::kStages + 9);
  float* parts = (float*)(rest + C::kSwapBytes + C::kCountBytes + 512);   // [rank - 1][row][feature]
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool PAIR = C::PAIR;
  const int place = SHARE == kAlone ? 0 : (int)cluster_rank(), rank = PAIR ? place : 0;
  // dweight: a group's last slab is complete when a warp of its own has cleared the rows of the next group in it, in each CTA
  constexpr bool kTail = KIND == kDweight;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar_full + 8 * s, kTail ? C::kCtas : 1);
      mbar_init(bar_empty + 8 * s, 1);
      mbar_init(bar_tail + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(bar_tfull + 8 * b, 1);
      mbar_init(bar_tempty + 8 * b, C::kEpilogueWarps * C::kCtas);
    }
    for (int b = 0; b < 4; ++b) mbar_init(bar_swap + 8 * b, 2);
    mbar_init(bar_parts, SHARE == kSplit ? (cluster_size() - 1) * C::kEpilogueWarps : 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (SHARE != kAlone) cluster_sync();
  if (warp == 1) take_tmem<PAIR>(smem_u32(tmem_slot), 2 * BN);
  after_previous();
  if (KIND != kDweight) count_tiles(p.groups, BN, before, before + p.groups.G + 1);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const Walk<KIND, GATED, BN, SHARE> walk(p, before);

  Item it, mine;
  if (warp == 0) {
    uint32_t stage = 0, phase = 0;
    bool alive = true;
    for (int i = 0; alive && walk.at(i, mine, it); ++i) {
      if (lane == 0) {
        const int slabs = walk.slabs(it), part = GATED && KIND == kBackward ? slabs / 2 : slabs;
        const int f0 = it.f0 + rank * (C::kFeatures / C::kCtas);
        // this CTA's share of the MMA's N dimension
        const int share = walk.wide(it) / C::kCtas;
        const int row = it.row + rank * share, j0 = it.j0 + rank * share;
        const int panels = KIND == kDweight && maps.b_whole ? 2 : (share + 63) / 64;
        // a CTA's rows come in one copy of the lowest box that has them: a second copy costs more than the rows that it saves
        constexpr int kQuarter = C::kRowBox / 4;
        const int quarters = (share + kQuarter - 1) / kQuarter;
        const uint32_t part_b = quarters * kQuarter * 128;
        int from, to;
        walk.range(it, place, from, to);
        for (int kt = from; kt < to; ++kt) {
          if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, &wait_error, 1u)) {
            alive = false;
            break;
          }
          const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + C::kABytes;
          const int left = it.rows - kt * C::kSlab;             // dweight: rows of the group from here on
          const int low = KIND == kDweight && left <= 64;       // they come in the lower box
          const uint32_t panel = (low ? 64 : C::kSlab) * 128;   // of an operand across its rows
          const uint32_t tx = KIND == kDweight ? (2 + panels) * panel : C::kABytes + part_b;
          uint32_t full = bar_full + 8 * stage;
          const bool tail = kTail && left < C::kSlab;
          if (tail) {
            full = bar_tail + 8 * stage;   // waited for by this CTA's clearing warp, which then arrives at the leader's barrier
            mbar_expect_tx(full, tx);
          } else if (rank == 0) {
            mbar_expect_tx(full, C::kCtas * tx);
          } else {
            full = leaders(full);
            if (kTail) arrive_at_relaxed(full);   // the copies themselves say when they have landed
          }
          if (KIND == kForward) {
            const int x = kt * C::kSlab;
            if (maps.a_whole) {
              const int y = it.g * maps.a_step + f0;
              load_2d<PAIR>(sa, &maps.a[0], x, y, full);
              if (GATED) load_2d<PAIR>(sa + C::kABytes / 2, &maps.a_up[0], x, y, full);
            } else {
              load_3d<PAIR>(sa, &maps.a[0], x, f0, it.g, full);
              if (GATED) load_3d<PAIR>(sa + C::kABytes / 2, &maps.a_up[0], x, f0, it.g, full);
            }
            load_2d<PAIR>(sb, &maps.b[quarters - 1], x, row, full);
          } else if (KIND == kBackward) {
            const bool up = kt >= part;
            const int x = (up ? kt - part : kt) * C::kSlab;
            load_panels<PAIR>(sa, up ? &maps.a_up[0] : &maps.a[0], maps.a_whole, 2, panel, f0, x, it.g, full);
            load_2d<PAIR>(sb, up ? &maps.b_up[quarters - 1] : &maps.b[quarters - 1], x, row, full);
          } else {
            const int y = it.row + kt * C::kSlab;
            load_panels<PAIR>(sa, it.half ? &maps.a_up[low] : &maps.a[low], maps.a_whole, 2, panel, f0, y, 0, full);
            load_panels<PAIR>(sb, &maps.b[low], maps.b_whole, panels, panel, j0, y, 0, full);
          }
          if (++stage == C::kStages) stage = 0, phase ^= 1u;
        }
      }
      alive = __shfl_sync(0xffffffffu, alive, 0);
    }
  } else if (warp == 1) {
    const uint64_t a_first = KIND == kForward ? smem_desc(smem_base) : smem_desc_across(smem_base, C::kSlab * 128);
    const uint64_t b_first = KIND == kDweight ? smem_desc_across(smem_base + C::kABytes, C::kSlab * 128) : smem_desc(smem_base + C::kABytes);
    uint32_t stage = 0, phase = 0, acc = 0;
    bool alive = rank == 0;   // the leader's MMAs are the pair's
    for (int i = 0; alive && walk.at(i, mine, it); ++i) {
      int from, to;
      walk.range(it, place, from, to);
      if (from == to) continue;
      const int cols = walk.wide(it);
      // fp32 sums of bf16, M = 128 (256 in a pair), N; a set bit 15 / 16: A / B lies across its rows
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)cols >> 3 << 17) | ((uint32_t)(kTileM * C::kCtas) >> 4 << 24) |
                             (KIND != kForward ? 1u << 15 : 0u) | (KIND == kDweight ? 1u << 16 : 0u);
      const uint32_t buf = acc & 1u;
      if (!warp_wait(bar_tempty + 8 * buf, ((acc >> 1) & 1u) ^ 1u, abort_flag, &wait_error, 2u)) break;
      ++acc;
      tc_fence_after();
      const uint32_t d = tmem_base + buf * BN;
      bool ok = true;   // one answer per tile, as in warp_wait (asked for every slab it cost a large product 2 %); after a "no" the slabs pass idly
      for (int kt = from; kt < to; ++kt) {
        ok = ok && mbar_wait(bar_full + 8 * stage, phase, abort_flag, &wait_error, 3u);
        const int left = KIND == kDweight ? it.rows - kt * C::kSlab : C::kSlab;
        tc_fence_after();
        if (lane == 0 && ok) {
          const uint64_t ad = a_first + stage * (C::kStageBytes >> 4), bd = b_first + stage * (C::kStageBytes >> 4);
          // from one 16 of the reduction to the next: 32 bytes along a swizzled row, 16 rows across
          constexpr uint32_t kStepA = (KIND == kForward ? 32 : 2048) >> 4, kStepB = (KIND == kDweight ? 2048 : 32) >> 4;
          if (left >= C::kSlab) {
#pragma unroll
            for (int k = 0; k < C::kSlab / 16; ++k) mma<PAIR>(d, ad + k * kStepA, bd + k * kStepB, idesc, ((kt - from) | k) != 0 ? 1u : 0u);
          } else {
            const uint64_t low = left <= 64 ? (uint64_t)(64 * 128 >> 4) << 16 : 0;   // panels half as far apart
            for (int k = 0; k < (left + 15) / 16; ++k) mma<PAIR>(d, ad - low + k * kStepA, bd - low + k * kStepB, idesc, ((kt - from) | k) != 0 ? 1u : 0u);
          }
          commit<PAIR>(bar_empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == C::kStages) stage = 0, phase ^= 1u;
      }
      alive = __all_sync(0xffffffffu, ok);
      if (alive && lane == 0) commit<PAIR>(bar_tfull + 8 * buf);
      __syncwarp();
    }
  } else if (kTail && warp == C::kClearWarp) {
    // Clears, in a group's last slab, the rows of the next group up to the next multiple of 16 (the MMAs go no further), of both operands: zero times
    // a NaN of the next group would not be zero.  In the MMAs' own warp this cost the 8 slabs of a group of 500 rows 20 us of 300.
    uint32_t stage = 0, tails = 0;   // tails: the phase of every stage's bar_tail
    int64_t since = 0;               // slabs multiplied since this warp last had one to clear
    for (int i = 0; walk.at(i, mine, it); ++i) {
      const int slabs = walk.slabs(it), valid = it.rows - (slabs - 1) * C::kSlab;
      if (slabs == 0) continue;
      since += slabs;
      stage = (stage + slabs - 1) % C::kStages;
      if (valid < C::kSlab) {
        if (!warp_wait(bar_tail + 8 * stage, (tails >> stage) & 1u, abort_flag, &wait_error, 6u, reduction_limit_ns(since))) break;
        since = 0;
        tails ^= 1u << stage;
        // a row's 128 bytes in two panels of dout and two of x at a time
        const int panel = (valid <= 64 ? 64 : C::kSlab) * 128;
        uint8_t* at = smem_al + (size_t)stage * C::kStageBytes + (lane >> 4) * C::kABytes + (lane >> 3 & 1) * panel + (lane & 7) * 16;
        for (int r = valid; r & 15; ++r) *(uint4*)(at + r * 128) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          // The leader's MMAs read this CTA's rows, so rank 1 arrives with a cluster-wide release: 20 us of 254 at 64 groups of 500 rows, but a
          // relaxed arrival would leave the clearing unordered.  Copies of 16 rows and of one, zeros from behind the operand's end, took 353.
          if (rank != 0) arrive_at(leaders(bar_full + 8 * stage));
          else mbar_arrive(bar_full + 8 * stage);
        }
      }
      stage = (stage + 1) % C::kStages;
    }
  } else {
    const int quad = warp & 3, team = (warp - 2) >> 2;   // TMEM lanes this warp may read; which chunks it takes
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    uint32_t acc = 0, swaps = 0;
    bool alive = true;
    for (int i = 0; alive && walk.at(i, mine, it); ++i) {
      it.f0 += rank * (C::kFeatures / C::kCtas);
      int from, to;
      walk.range(it, place, from, to);
      const bool sums = to > from;
      const uint32_t buf = acc & 1u;
      // what the layer below kept is asked for a chunk ahead, the first before the sums are there
      Backward<__nv_bfloat16>::Asked<1> asked;
      if constexpr (KIND == kBackward)
        Backward<__nv_bfloat16>(p.bwd, it.g, it.f0 + quad * 32 + 8 * (lane & 3)).ask((int64_t)it.row + 8 * team, it.rows - 8 * team, asked);
      if (sums) {
        if (!warp_wait(bar_tfull + 8 * buf, (acc >> 1) & 1u, abort_flag, &wait_error, 4u, reduction_limit_ns(to - from))) break;
        ++acc;
        tc_fence_after();
      }
      const uint32_t t0 = tmem_base + lane_addr + buf * BN;
      if constexpr (SHARE == kSplit) {
        // At most one tile per cluster.  The others hand their sums to rank 0, which adds them in the order of their ranks.
        if (place != 0) {
          const uint32_t to0 = leaders(smem_u32(parts + (size_t)(place - 1) * BN * kTileM + quad * 32 + lane));
          for (int c = 8 * team; c < walk.wide(it); c += 8 * C::kTeams) {
            float v[8] = {};
            __syncwarp();
            if (sums) {
              tmem_ld8(t0 + c, v);
              tmem_ld_wait();
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
              asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to0 + (uint32_t)((c + j) * kTileM * 4)), "f"(v[j]) : "memory");
          }
          __syncwarp();
          if (lane == 0) arrive_at(leaders(bar_parts));
          break;
        }
        if (cluster_size() > 1 && !warp_wait_cluster(bar_parts, 0u, abort_flag, &wait_error, 7u, reduction_limit_ns(to - from))) break;
      }
      auto add_parts = [&](auto& v, int c) {
        if constexpr (SHARE == kSplit) {
          for (int r = 1; r < (int)cluster_size(); ++r)
#pragma unroll
            for (int j = 0; j < (int)(sizeof(v) / 4); ++j) v[j] += parts[((size_t)(r - 1) * BN + c + j) * kTileM + quad * 32 + lane];
        }
      };
      if constexpr (KIND == kDweight) {
        const int cols = min(BN, p.k - it.j0), first_row = it.f0 + quad * 32;
        const void* add = it.half ? p.add_dw_up : p.add_dw;
        void* dw = it.half ? p.dw_up : p.dw;
        const int64_t at = it.g * p.step_w + (int64_t)first_row * p.ld_w + it.j0;
        uint8_t* buffer = (uint8_t*)swap + (warp - 2) * 4096;
        if (maps.d_copies && first_row < p.n) {
          // whole lines, written by copies of 32 rows x 128 bytes from shared memory, which cut off what lies outside the matrix
          const CUtensorMap* map = it.half ? &maps.d_up : &maps.d;
          const int per = p.dw_f32 ? 32 : 64;
          for (int c = per * team; c < cols; c += 2 * per) {
            float v[32] = {};
            uint32_t w[32];
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
            if (sums) {
              tmem_ld32(t0 + c, v);
              tmem_ld_wait();
            }
            if (p.dw_f32) {
#pragma unroll
              for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(v[j]);
            } else {
              float u[32] = {};
              if (sums && c + 32 < BN) {
                tmem_ld32(t0 + c + 32, u);
                tmem_ld_wait();
              }
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]), b = __floats2bfloat162_rn(u[2 * j], u[2 * j + 1]);
                w[j] = *(const uint32_t*)&a, w[16 + j] = *(const uint32_t*)&b;
              }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *(uint4*)(buffer + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(buffer)),
                           "r"(it.j0 + c), "r"(first_row), "r"(it.g)
                           : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          }
        } else if (first_row < p.n) {
          for (int c = 32 * team; c < cols; c += 64) {
            float v[32] = {};
            __syncwarp();   // the loads from TMEM take the whole warp
            if (sums) {
              tmem_ld32(t0 + c, v);
              tmem_ld_wait();
            }
            typedef __nv_bfloat16 B;
            const int rows = p.n - first_row;
            if (p.dw_f32) store_block(buffer, v, (float*)dw + at + c, add ? (const float*)add + at + c : nullptr, p.ld_w, rows, cols - c, p.dw_wide);
            else store_block(buffer, v, (B*)dw + at + c, add ? (const B*)add + at + c : nullptr, p.ld_w, rows, cols - c, p.dw_wide);
          }
        }
      } else if constexpr (KIND == kForward && GATED) {
        // quadrants 0 and 1 hold z, 2 and 3 z_up of the same 64 features; of every 16 rows the first 8 are finished by the warp that holds z
        const int pair = (quad & 1) * 2 + team, up = (quad >> 1);
        const Forward<__nv_bfloat16, true> e(p.fwd, it.g, it.f0 + (quad & 1) * 32 + 8 * (lane & 3));
        for (int c = 16 * team; c < it.rows; c += 32, ++swaps) {
          float v[16], z[1][8], z_up[1][8];
          __syncwarp();
          tmem_ld16(t0 + c, v);
          tmem_ld_wait();
          add_parts(v, c);
          float* both = swap + (pair * 2 + (swaps & 1)) * 2 * 16 * kSwapStride;
#pragma unroll
          for (int j = 0; j < 16; ++j) both[(up * 16 + j) * kSwapStride + lane] = v[j];
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_swap + 8 * pair);
          if (!warp_wait(bar_swap + 8 * pair, swaps & 1u, abort_flag, &wait_error, 5u)) {
            alive = false;
            break;
          }
          row_of(both, up * 8, z[0]);
          row_of(both + 16 * kSwapStride, up * 8, z_up[0]);
          e.rows((int64_t)it.row + c + up * 8, it.rows - c - up * 8, z, z_up);
        }
      } else {
        typedef typename std::conditional<KIND == kForward, Forward<__nv_bfloat16, false>, Backward<__nv_bfloat16>>::type Epilogue;
        typename std::conditional<KIND == kForward, const ForwardArgs&, const BackwardArgs&>::type args = [&]() -> auto& {
          if constexpr (KIND == kForward) return p.fwd;
          else return p.bwd;
        }();
        const Epilogue e(args, it.g, it.f0 + quad * 32 + 8 * (lane & 3));
        float* turn = swap + (warp - 2) * 8 * kSwapStride;
        for (int c = 8 * team; c < it.rows; c += 8 * C::kTeams) {
          float v[8], t[1][8];
          const Backward<__nv_bfloat16>::Asked<1> q = asked;
          if constexpr (KIND == kBackward) e.ask((int64_t)it.row + c + 8 * C::kTeams, it.rows - c - 8 * C::kTeams, asked);
          __syncwarp();
          tmem_ld8(t0 + c, v);
          tmem_ld_wait();
          add_parts(v, c);
#pragma unroll
          for (int j = 0; j < 8; ++j) turn[j * kSwapStride + lane] = v[j];
          __syncwarp();
          row_of(turn, 0, t[0]);
          if constexpr (KIND == kBackward) {
            e.rows((int64_t)it.row + c, it.rows - c, t, q);
          } else {
            float none[1][8];
            e.rows((int64_t)it.row + c, it.rows - c, t, none);
          }
        }
      }
      if (sums) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) arrive_at_relaxed(leaders(bar_tempty + 8 * buf));   // the sums are in registers; the stores need not have landed
          else mbar_arrive(bar_tempty + 8 * buf);
        }
      }
    }
  }

  if (KIND == kDweight && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncwarp();
  if (*abort_flag) {
    // copies and MMAs still in flight land before shared memory and TMEM are released
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (SHARE != kAlone) cluster_sync();   // no CTA leaves while another may still reach its shared memory
  tc_fence_after();
  if (warp == 1) free_tmem<PAIR>(tmem_base, 2 * BN);
}

constexpr int64_t kMostStride = 1ll << 38;   // elements: a tensor map's strides are below 2^40 bytes

// ---- host ---------------------------------------------------------------------------------------------------------
bool encode(CUtensorMap* m, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
            CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16) {
  const cuuint32_t one[4] = {1, 1, 1, 1};
  EncodeFn fn = encode_fn();
  return fn && fn(m, type, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [rows, cols] read along its rows: boxes of 64 columns and 1/4 .. 4/4 of `most` rows
bool map_rows(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  return encode(m, base, 2, dims, strides, box);
}
bool map_boxes(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t ld, int most) {
  for (int i = 0; i < 4; ++i)
    if (!map_rows(m + i, base, rows, cols, ld, most / 4 * (i + 1))) return false;
  return true;
}
cuuint64_t matrix_step(int64_t matrices, int64_t rows, int64_t ld, int64_t step) {   // one matrix: any multiple of 16 bytes
  return (cuuint64_t)(matrices > 1 ? step : (rows * ld + 7) & ~7ll) * 2;
}
// [groups, n, k] read along its rows.  Rows behind a matrix's last may come from the next one: they are features that nobody stores.
bool map_weights(CUtensorMap* m, const void* base, const Problem& p, int box_rows, int* whole, int* step) {
  const int64_t apart = p.groups.G > 1 ? p.step_w / p.ld_w : p.n, rows = (p.groups.G - 1) * apart + p.n;
  *whole = (p.groups.G == 1 || p.step_w % p.ld_w == 0) && rows <= 0x7fffffffll;
  *step = (int)apart;
  if (*whole) return map_rows(m, base, rows, p.k, p.ld_w, box_rows);
  const cuuint64_t dims[3] = {(cuuint64_t)p.k, (cuuint64_t)p.n, (cuuint64_t)p.groups.G};
  const cuuint64_t strides[2] = {(cuuint64_t)p.ld_w * 2, matrix_step(p.groups.G, p.n, p.ld_w, p.step_w)};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return encode(m, base, 3, dims, strides, box);
}
bool whole(int64_t cols) { return cols % 64 == 0; }
// [matrices, rows, cols] read across its rows, `box_rows` at a time
bool map_panels(CUtensorMap* m, const void* base, int64_t matrices, int64_t rows, int64_t cols, int64_t ld, int64_t step, int box_rows) {
  const cuuint64_t sg = matrix_step(matrices, rows, ld, step);
  if (whole(cols)) {
    const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64), (cuuint64_t)matrices}, strides[3] = {(cuuint64_t)ld * 2, 128, sg};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 2, 1};
    return encode(m, base, 4, dims, strides, box);
  }
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)matrices}, strides[2] = {(cuuint64_t)ld * 2, sg};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return encode(m, base, 3, dims, strides, box);
}

// dw [groups, n, k], boxes of 32 rows x 128 bytes; false where its rows are not aligned to 16 bytes
bool map_dw(CUtensorMap* m, const void* base, const Problem& p) {
  const int e = p.dw_f32 ? 4 : 2;
  const cuuint64_t sg = p.groups.G > 1 ? (cuuint64_t)p.step_w * e : ((cuuint64_t)p.n * p.ld_w * e + 15) & ~(cuuint64_t)15;
  if (((uintptr_t)base | (uintptr_t)(p.ld_w * e) | (uintptr_t)sg) & 15 || p.ld_w >= kMostStride / 2 || sg >= (1ull << 40)) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)p.k, (cuuint64_t)p.n, (cuuint64_t)p.groups.G}, strides[2] = {(cuuint64_t)p.ld_w * e, sg};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / e), 32, 1};
  return encode(m, base, 3, dims, strides, box, p.dw_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16);
}
// Tiles of a product, at most
template <int KIND, bool GATED, int BN, int SHARE>
int64_t most_tiles(const Problem& p) {
  using C = Cfg<KIND, GATED, BN, SHARE>;
  const int64_t rows = p.L * p.groups.R, FT = ((KIND == kBackward ? p.k : p.n) + C::kFeatures - 1) / C::kFeatures;
  if (KIND == kDweight) return (int64_t)p.groups.G * (GATED ? 2 : 1) * FT * ((p.k + BN - 1) / BN);
  return (p.groups.G == 1 ? (rows + BN - 1) / BN : rows / BN + p.groups.G) * FT;
}
// CTAs per tile: as many as leave every cluster one tile and every CTA eight slabs.
int split_of(const Problem& p, int kind, int64_t tiles, int bn, int sms) {
  const int64_t slabs = (int64_t)((kind == kBackward ? p.n : p.k) + 63) / 64 * (kind == kBackward && p.gated ? 2 : 1);
  int s = most_parts(bn);
  while (s > 1 && (tiles * s > sms || slabs < 8 * s)) s /= 2;
  return s;
}

template <int KIND, bool GATED, int BN, int SHARE>
cudaError_t launch(const Problem& p, cudaStream_t st) {
  using C = Cfg<KIND, GATED, BN, SHARE>;
  static int cache[64] = {0}, pairs[64] = {0};
  auto kernel = linear_tc_kernel<KIND, GATED, BN, SHARE>;
  int sms = 0, dev = 0;
  cudaError_t e = sm_count_and_smem_optin(kernel, C::kSmemBytes, cache, &sms);
  if (e != cudaSuccess) return e;
  Maps m;
  bool ok;
  const int64_t rows = p.L * p.groups.R, most = most_tiles<KIND, GATED, BN, SHARE>(p);
  const __nv_bfloat16* y = (const __nv_bfloat16*)p.y;
  m.a_whole = m.b_whole = m.a_step = m.d_copies = 0;
  if (KIND == kDweight) {
    static_assert(KIND != kDweight || BN / C::kCtas == 128, "two panels of x's columns per CTA");
    m.a_whole = whole(p.n), m.b_whole = whole(p.k);
    m.d_copies = !p.add_dw && map_dw(&m.d, p.dw, p) && (!GATED || map_dw(&m.d_up, p.dw_up, p));
    ok = true;
    for (int i = 0; i < 2; ++i)
      ok = ok && map_panels(&m.a[i], y, 1, rows, p.n, p.ld_y, 0, 128 >> i) && map_panels(&m.b[i], p.x, 1, rows, p.k, p.ld_x, 0, 128 >> i) &&
           (!GATED || map_panels(&m.a_up[i], y + p.half_y, 1, rows, p.n, p.ld_y, 0, 128 >> i));
  } else if (KIND == kForward) {
    const int box = GATED ? kTileM / 2 : kTileM;
    ok = map_weights(&m.a[0], p.w, p, box, &m.a_whole, &m.a_step) && (!GATED || map_weights(&m.a_up[0], p.w_up, p, box, &m.a_whole, &m.a_step)) &&
         map_boxes(m.b, p.x, rows, p.k, p.ld_x, C::kRowBox);
  } else {
    m.a_whole = whole(p.k);
    ok = map_panels(&m.a[0], p.w, p.groups.G, p.n, p.k, p.ld_w, p.step_w, C::kSlab) &&
         (!GATED || map_panels(&m.a_up[0], p.w_up, p.groups.G, p.n, p.k, p.ld_w, p.step_w, C::kSlab));
    ok = ok && map_boxes(m.b, y, rows, p.n, p.ld_y, C::kRowBox) && (!GATED || map_boxes(m.b_up, y + p.half_y, rows, p.n, p.ld_y, C::kRowBox));
  }
  if (!ok || most > 0x7fffffffll) return cudaErrorInvalidValue;
  int ctas = C::kCtas;
  if (SHARE == kSplit) ctas = split_of(p, KIND, most, BN, sms);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = sms / ctas * ctas, cfg.blockDim = C::kThreads, cfg.dynamicSmemBytes = C::kSmemBytes, cfg.stream = st, cfg.attrs = attr, cfg.numAttrs = 2;
  int64_t units = sms;
  if (SHARE == kPair) {
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (!pairs[dev] && (e = cudaOccupancyMaxActiveClusters(&pairs[dev], kernel, &cfg)) != cudaSuccess) return e;
    units = pairs[dev] > 0 ? pairs[dev] : 1;
  }
  // several CTAs on a reduction: a cluster per tile
  cfg.gridDim = (unsigned)((SHARE == kSplit || most < units ? most : units) * ctas);
  return cudaLaunchKernelEx(&cfg, kernel, m, p);
}

// Rows per tile by the rows that a group has on average.  Where all tiles together leave half of the SMs idle, up to four CTAs share a tile's reduction (16 rows
// x 14336 x 4096, 32 tiles: 70 us alone, 27 shared); a pair of CTAs wants more rows than one (below 96 its tiles would be mostly empty).
// Tiles of 32 rows read fewer rows that belong to another group, tiles of 128 read the weights once; 60 groups, 2048 -> 1408, us with 32 / with 128, forward,
// gated forward, row gradient:    8 rows each 61 / 62, 104 / 108, 61 / 60    16: 61 / 63, 110 / 111, 61 / 61    24: 64 / 65, 123 / 113, 73 / 63
// 28: 73 / 65, 128 / 113, 74 / 65    40: 78 / 66, 155 / 121, 96 / 67.  (24 is the forward pass's border; gradients would take 16.)
template <int KIND, bool GATED>
cudaError_t launch_rows(const Problem& p, int sms, cudaStream_t st) {
  const int64_t each = p.L * p.groups.R / p.groups.G;
  if (each <= 32 && split_of(p, KIND, most_tiles<KIND, GATED, 32, kSplit>(p), 32, sms) > 1) return launch<KIND, GATED, 32, kSplit>(p, st);
  if (each > 32 && each <= 64 && split_of(p, KIND, most_tiles<KIND, GATED, 64, kSplit>(p), 64, sms) > 1)
    return launch<KIND, GATED, 64, kSplit>(p, st);
  if (each > 64 && each <= 256 && split_of(p, KIND, most_tiles<KIND, GATED, 128, kSplit>(p), 128, sms) > 1)
    return launch<KIND, GATED, 128, kSplit>(p, st);
  if (each <= 24) return launch<KIND, GATED, 32, kAlone>(p, st);
  if (each <= 96) return launch<KIND, GATED, 128, kAlone>(p, st);
  return launch<KIND, GATED, 256, kPair>(p, st);
}

bool tma_rows(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < kMostStride; }

// Waits, as the kernels' warps do, on a barrier that nothing arrives at; the wait gives up after limit_ns and is noted as theirs are.
__global__ void wait_selftest_kernel(unsigned long long limit_ns) {
  __shared__ uint64_t bar;
  __shared__ uint32_t abort_flag;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar), 1);
    abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  warp_wait(smem_u32(&bar), 0u, &abort_flag, &wait_error, 99u, limit_ns);
}

}  // namespace

bool tensor_applicable(Kind kind, const Problem& p, int32_t dtype) {
  if (dtype != MCCE_BF16) return false;
  if (kind == kDweight) return p.L * p.groups.R > 0 && tma_rows(p.y, p.ld_y) && tma_rows(p.x, p.ld_x) && (!p.gated || p.half_y % 8 == 0);
  if (!tma_rows(p.w, p.ld_w) || !tma_rows(p.w_up, p.ld_w) || (p.groups.G > 1 && (p.step_w % 8 || p.step_w >= kMostStride))) return false;
  if (kind == kForward) return tma_rows(p.x, p.ld_x);
  return tma_rows(p.y, p.ld_y) && (!p.gated || p.half_y % 8 == 0);
}

cudaError_t run_tensor(Kind kind, const Problem& p, cudaStream_t st) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaErrorInvalidDevice;
  if (kind == kForward) return p.gated ? launch_rows<kForward, true>(p, sms, st) : launch_rows<kForward, false>(p, sms, st);
  if (kind == kBackward) return p.gated ? launch_rows<kBackward, true>(p, sms, st) : launch_rows<kBackward, false>(p, sms, st);
  return p.gated ? launch<kDweight, true, 256, kPair>(p, st) : launch<kDweight, false, 256, kPair>(p, st);
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

extern "C" int mcce_selftest_expert_linear_timeout(uint64_t limit_ns, void* cuda_stream) {
  if (limit_ns == 0 || limit_ns > 1000000000ull) return MCCE_EINVAL;
  mcce::linear::wait_selftest_kernel<<<1, 64, 0, (cudaStream_t)cuda_stream>>>(limit_ns);
  return cudaGetLastError() == cudaSuccess ? MCCE_OK : MCCE_ECUDA;
}
