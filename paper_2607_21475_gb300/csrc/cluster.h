// Size of a cluster beyond the portable eight CTAs, where the GPU has room for it.
#pragma once

#include <atomic>

namespace ebd {

constexpr int kPortableCluster = 8, kClusterDevices = 64;

// Whether a kernel's clusters of its largest size were found to fit, per device (0: not asked).
struct ClusterMemo {
  std::atomic<signed char> fits[kClusterDevices] = {};
};

// `want` CTAs, or 8 where that is more and no cluster of the kernel's largest size can run, as
// on a partition of a GPU whose groups of SMs are smaller: how many can is what active() says
// (none: also where it fails), asked once per device.
template <typename Active>
int cluster_ctas(int want, ClusterMemo& memo, int device, Active active) {
  if (want <= kPortableCluster) return want;
  if (device < 0 || device >= kClusterDevices) return kPortableCluster;
  signed char fits = memo.fits[device].load(std::memory_order_relaxed);
  if (fits == 0) {
    fits = active() > 0 ? 1 : -1;
    memo.fits[device].store(fits, std::memory_order_relaxed);
  }
  return fits > 0 ? want : kPortableCluster;
}

}  // namespace ebd
