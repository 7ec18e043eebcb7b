// experts_device.h -- which expert's rows a workgroup of the grouped products
// takes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mxq_internal.h"

namespace mxq {

// Inclusive sums over the wave's lanes (row shifts, then the rows' last lanes).
__device__ inline int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// The experts' rows in tiles of 2^LG, an expert's last one shorter (a multiple of
// 16): tile i is rows row0 .. row0 + rows - 1 of expert e; rows 0 behind the last.
// Every lane of the wave calls it.
struct ExpertTile {
  int e, row0, rows;
};
template <int LG>
__device__ inline ExpertTile expert_tile(const Groups &x, int i) {
  const int lane = threadIdx.x & 63;
  for (int b = 0; b < x.E; b += 64) {
    const int e = b + lane;
    const int lo = x.first[min(e, x.E)], hi = x.first[min(e + 1, x.E)];
    const int n = (hi - lo + (1 << LG) - 1) >> LG, upto = wave_scan(n);
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (i < all) {
      const int l = __builtin_ctzll(__ballot(upto > i));
      const int at = i - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
      ExpertTile t;
      t.e = b + l;
      t.row0 = __builtin_amdgcn_readlane(lo, l) + (at << LG);
      t.rows = min(1 << LG, __builtin_amdgcn_readlane(hi, l) - t.row0);
      if (t.row0 < 0 || t.row0 + (int64_t)t.rows > x.rows) break;   // (not a plan)
      return t;
    }
    i -= all;
  }
  return ExpertTile{0, 0, 0};
}

}  // namespace mxq
