// What the kernels of the experts' products and of their gradients share: the map of the slots' tiles, and two types.
#pragma once

#include "eep_internal.hpp"
#include "numbers.hpp"

namespace eep {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) void lds_void;

// The tiles of the slots: what one wavefront has to remember to find any of them.  Args has the offsets (NULL: one slot), rows,
// slots and feature_tiles.
template <int TOKENS>
struct TileMap {
  int run;   // slots a lane counts
  int upto;  // tiles of the slots up to the end of this lane's run
  int total;

  __device__ __forceinline__ static int tiles_of(int lo, int hi) { return hi > lo ? (hi - lo + TOKENS - 1) / TOKENS : 0; }
  template <class Args>
  __device__ __forceinline__ static int bound(const Args& a, int p) {
    const int o = a.offset[p];
    return o < 0 ? 0 : o > a.rows ? a.rows : o;
  }
  __device__ __forceinline__ static int running_sum(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int other = __shfl_up(v, d, 64);
      if (lane >= d) v += other;
    }
    return v;
  }

  template <class Args>
  __device__ __forceinline__ void make(const Args& a) {
    if (a.offset == nullptr) {
      total = tiles_of(0, a.rows);
      return;
    }
    const int lane = threadIdx.x & 63;
    run = (a.slots + 63) / 64;
    const int p0 = lane * run, p1 = p0 + run < a.slots ? p0 + run : a.slots;
    int mine = 0;
    if (p0 < p1) {
      int lo = bound(a, p0);
      for (int p = p0; p < p1; ++p) {
        const int hi = bound(a, p + 1);
        mine += tiles_of(lo, hi);
        lo = hi;
      }
    }
    upto = running_sum(mine);
    total = __builtin_amdgcn_readlane(upto, 63);
  }

  // Item `item` of total * feature_tiles: slot, feature tile, first row and the end of the slot's rows.
  template <class Args>
  __device__ __forceinline__ void find(const Args& a, int64_t item, int* slot, int* feature_tile, int* first,
                                       int* end) const {
    if (a.offset == nullptr) {
      *slot = 0;
      *feature_tile = (int)(item / total);
      *first = (int)(item - (int64_t)*feature_tile * total) * TOKENS;
      *end = a.rows;
      return;
    }
    const int lane = threadIdx.x & 63;
    const int owner = __builtin_ctzll(__ballot((int64_t)upto * a.feature_tiles > item));
    int before = owner > 0 ? __builtin_amdgcn_readlane(upto, owner - 1) : 0;
    for (int p0 = owner * run;; p0 += 64) {
      // the lanes look at 64 slots of the run; the item is in one of the run's
      const int p = p0 + lane;
      const bool in = p < (owner + 1) * run && p < a.slots;
      const int lo = in ? bound(a, p) : 0, hi = in ? bound(a, p + 1) : 0;
      const int tiles = tiles_of(lo, hi);
      const int sum = before + running_sum(tiles);
      const uint64_t behind = __ballot((int64_t)sum * a.feature_tiles > item);
      if (behind != 0) {
        const int who = __builtin_ctzll(behind);
        const int n = __builtin_amdgcn_readlane(tiles, who);
        const int left = (int)(item - (int64_t)(__builtin_amdgcn_readlane(sum, who) - n) * a.feature_tiles);
        *slot = p0 + who;
        *feature_tile = left / n;
        *first = __builtin_amdgcn_readlane(lo, who) + (left - *feature_tile * n) * TOKENS;
        *end = __builtin_amdgcn_readlane(hi, who);
        return;
      }
      if (p0 + 64 >= (owner + 1) * run) {  // (offsets that changed while the kernel ran)
        *slot = *feature_tile = *first = *end = 0;
        return;
      }
      before = __builtin_amdgcn_readlane(sum, 63);
    }
  }
};

}  // namespace eep
