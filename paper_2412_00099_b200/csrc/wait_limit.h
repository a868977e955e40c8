// Host and device: how long a bounded wait of the tensor-core kernels may last.
#pragma once
#ifdef __CUDACC__
#define MCCE_HOST_DEVICE __host__ __device__
#else
#define MCCE_HOST_DEVICE
#endif

namespace mcce {
namespace tc {

constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // every mbarrier wait gives up after 2 s
constexpr unsigned long long kSlabLimitNs = 20000ull;        // a slab of a reduction takes 0.4 to 0.8 us

// A wait that lasts as long as the products of a tile, or of several, do: `slabs` is all that may be multiplied while it lasts (2^31 - 1 rows are
// 2^24 slabs, some 10 s).
MCCE_HOST_DEVICE constexpr unsigned long long reduction_limit_ns(long long slabs) {
  return kWaitLimitNs + kSlabLimitNs * (unsigned long long)(slabs > 0 ? slabs : 0);
}

}  // namespace tc
}  // namespace mcce
