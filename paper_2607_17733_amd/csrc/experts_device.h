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

// The experts' rows in tiles of 2^LG rows (an expert's last one shorter, a multiple of
// 16), each with `ntiles` column tiles.  Workgroup pid takes rows row0 .. row0 + rows -
// 1 of expert e and column tile nt; rows 0: nothing is left for it.
//
// The tiles lie in order of the experts, `near` row tiles to a column tile; groups of
// `near` go to the XCDs (workgroup pid to pid % 8) in turn, so that all have as many and
// surplus workgroups come last.  (An eighth of all tiles in one run for each XCD was 8 %
// faster, 2048 tokens down 67 against 73 us, to 50 % slower, 333 tokens 42 against 28;
// column tiles bound to XCDs, whose number is no multiple of 8, 55 against 48 for 64 tokens
// among 128 experts.)  Every lane of the wave calls it.
struct ExpertTile {
  int e, row0, rows, nt;
};
template <int LG>
__device__ inline ExpertTile expert_tile(const Groups &x, int pid, int ntiles, int near) {
  const int lane = threadIdx.x & 63;
  constexpr int kAhead = 4;                                // 256 experts' bounds in one latency
  int lo[kAhead], hi[kAhead];
  auto bounds = [&](int b0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = b0 + 64 * k + lane;
      lo[k] = x.first[min(e, x.E)];
      hi[k] = x.first[min(e + 1, x.E)];
    }
  };
  auto tiles = [&](int k) { return (hi[k] - lo[k] + (1 << LG) - 1) >> LG; };
  const ExpertTile none = {0, 0, 0, 0};
  const int loc = pid >> 3, q = loc / near, u = 8 * q + (pid & 7);
  int i = near * (u / ntiles) + loc - near * q;
  for (int b0 = 0; b0 < x.E; b0 += 64 * kAhead) {
    bounds(b0);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (b0 + 64 * k >= x.E) break;
      const int n = tiles(k), upto = wave_scan(n);
      const int all = __builtin_amdgcn_readlane(upto, 63);
      if (i < all) {
        const int l = __builtin_ctzll(__ballot(upto > i));
        const int at = i - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
        ExpertTile t;
        t.e = b0 + 64 * k + l;
        t.row0 = __builtin_amdgcn_readlane(lo[k], l) + (at << LG);
        t.rows = min(1 << LG, __builtin_amdgcn_readlane(hi[k], l) - t.row0);
        t.nt = u % ntiles;
        if (t.row0 < 0 || t.row0 + (int64_t)t.rows > x.rows) return none;   // (no plan)
        return t;
      }
      i -= all;
    }
  }
  return none;
}

}  // namespace mxq
