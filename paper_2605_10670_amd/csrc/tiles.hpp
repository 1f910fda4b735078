// What the kernels of the experts' products and of their gradients share: operands of the matrix cores, stores of their
// results, the map of the slots' tiles.
#pragma once

#include "eep_internal.hpp"
#include "numbers.hpp"

namespace eep {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;  // along in_features

// 32 bytes a lane of a 16-row operand: two chunks of 16.
struct Frag {
  u32x4 c[2];
};

// acc + a * b over the 128 bytes of a step.
template <int DT>
__device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 acc) {
  if constexpr (DT == EEP_BF16) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.c[j]),
                                                    __builtin_bit_cast(bf16x8, b.c[j]), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.c[j][i]), __uint_as_float(b.c[j][i]), acc, 0, 0, 0);
  }
  return acc;
}

// Stores four neighbouring features of one token.
template <int YT>
__device__ __forceinline__ void store4(uint8_t* y, int64_t element, const float (&v)[4]) {
  if constexpr (YT == EEP_F32)
    *(f32x4*)(y + element * 4) = f32x4{v[0], v[1], v[2], v[3]};
  else
    *(u32x2*)(y + element * 2) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// Two tiles of 16 features side by side, of which a lane has four neighbouring ones each, as bf16: rows of lanes exchange halves,
// so that each has 16 bytes, the lanes of a row 64 at once: of feature (part & 1) * 16 + (part >> 1) * 8 on.
__device__ __forceinline__ u32x4 side_by_side(const f32x4& a, const f32x4& b) {
  const auto low = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[0], a[1]), pack_bf16x2(b[0], b[1]), false, false);
  const auto high = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[2], a[3]), pack_bf16x2(b[2], b[3]), false, false);
  return u32x4{low[0], high[0], low[1], high[1]};
}

// n: the first of the 32 features.
__device__ __forceinline__ void store_tiles(uint8_t* y, int64_t row, int features, int n, int part, bool in_rows,
                                            const f32x4& a, const f32x4& b) {
  const u32x4 v = side_by_side(a, b);
  n += (part & 1) * 16 + (part >> 1) * 8;
  if (in_rows && n < features) *(u32x4*)(y + (row * features + n) * 2) = v;
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

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
