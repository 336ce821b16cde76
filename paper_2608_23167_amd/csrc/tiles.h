// Device helpers shared by the tiled products.
#pragma once

#include "common.h"

namespace ssm {

// Tile order: the grid is 1-D over (split, n-tile, m-tile) triples.
// Workgroups are dealt to the 8 XCDs round-robin by linear id, so id w runs
// on XCD w % 8; the order below gives each XCD a contiguous range of the
// triples, split-major, then n-tiles, m-tiles innermost.  The workgroups that
// share a weight tile then run on the same XCD at about the same time and
// read it once into that XCD's L2, and each XCD touches as few K-slices of
// the activations as possible, so that its slice stays resident in its L2.
__device__ __forceinline__ void tile_of(int w, int total, int ntm, int mt, int& split, int& tn,
                                        int& tm) {
  const int per = total / 8;
  const int v = w < per * 8 ? (w % 8) * per + (w / 8) : w;
  split = v / ntm;
  const int t = v % ntm;
  tn = t / mt;
  tm = t % mt;
}

// Waits until at most N vector-memory operations of this wave are in flight.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// A workgroup barrier that waits for nothing else and that no access moves across.
__device__ __forceinline__ void pp_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A workgroup barrier once this wave's LDS accesses are done; its loads from memory
// stay in flight.
__device__ __forceinline__ void lds_written_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace ssm
