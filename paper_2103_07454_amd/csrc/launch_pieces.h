// Launches of more workgroups than one grid takes.
#pragma once
#include <stdint.h>

namespace evg {

// HIP takes fewer than 2^32 threads in a grid.  launch(first, groups) is called for each piece; kernels count their workgroups from `first` on.
// Whole rounds of the eight XCDs, so that a workgroup's is the same as in one grid.
template <typename Launch>
inline void launch_pieces(uint64_t groups, uint32_t threads, Launch launch) {
  const uint64_t most = 0xFFFFFFFFull / threads / 8 * 8;
  for (uint64_t first = 0; first < groups; first += most) launch((uint32_t)first, (uint32_t)(groups - first < most ? groups - first : most));
}

}  // namespace evg
