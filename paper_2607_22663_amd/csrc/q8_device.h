// Device helpers of the 8-bit cache's kernels: sums across a wave's lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mbe {
namespace {

// Sum over the lanes up to this one, by DPP: within rows of 16, then across.
__device__ inline uint32_t scan_lanes(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row_bcast:15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
// Largest over the lanes up to this one.
__device__ inline uint32_t max_lanes(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true)));
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false)));
  return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false)));
}
__device__ inline uint32_t lane_value(uint32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Rows of a ragged input before sequence b: the lengths before it, within [0,
// max_len], each.  Every lane of a wave must call.
__device__ inline int64_t rows_before(const int32_t *lens, int b, int max_len) {
  uint32_t rows = 0;
  for (int j0 = 0; j0 < b; j0 += 64) {
    const int j = j0 + static_cast<int>(threadIdx.x & 63);
    rows += lane_value(scan_lanes(j < b ? min(max(lens[j], 0), max_len) : 0), 63);
  }
  return rows;
}

}  // namespace
}  // namespace mbe
