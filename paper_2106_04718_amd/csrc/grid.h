// Launches of any number of workgroups.
#pragma once

#include <hip/hip_runtime.h>

namespace fs {

// A dimension of a launch holds fewer than 2^32 lanes, 2^24 workgroups of 256, and the
// runtime does not refuse more: it launches what 32 bits leave of their number.  So the
// workgroups are numbered along rows of kGridRow, and the last row's may number more
// than were asked for: the kernel lets these go.
constexpr unsigned kGridRow = 1u << 20;   // of at most 1024 lanes each; below 2^32 workgroups in all

inline dim3 wide_grid(long long workgroups) {
    if (workgroups <= kGridRow) return dim3((unsigned)workgroups);
    return dim3(kGridRow, (unsigned)((workgroups + kGridRow - 1) / kGridRow));
}

// Kernels that number their workgroups along one dimension: whether that holds them.
inline bool one_dimension(long long workgroups, unsigned lanes) { return workgroups * lanes <= 0xffffffffll; }

__device__ __forceinline__ unsigned wide_index() { return blockIdx.y * kGridRow + blockIdx.x; }

}  // namespace fs
