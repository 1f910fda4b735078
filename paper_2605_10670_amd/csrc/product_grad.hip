// The gradients of the experts' products: of the rows, of every slot's weights, and of the gate between.
//
// Both products have an operand whose rows lie across the sum: the weights, whose in_features are neighbours while the sum goes
// over their rows; and for the weights' gradient both, since that sum goes over tokens.  Such an operand goes through LDS as it lies in
// memory, a step of 128 bytes' worth of the sum deep, and is turned on the way to the registers: ds_read_b64_tr_b16 gives a lane four
// values of ONE column from four rows (fp32 values are read one by one).  What a lane holds then is what product.hip's kernels have:
// lane l has row (column) l % 16 and terms 16 * (l / 16) bytes into each half step.
#include <new>
#include <type_traits>

#include "eep_internal.hpp"
#include "numbers.hpp"
#include "tiles.hpp"

struct eep_product_grad {
  eep_product_grad_config cfg;
  int64_t slot_stride, grad_stride;  // bytes
  int cus;                           // of the device
};

namespace eep {

// ---------------------------------------------------------------------------
// the gate's gradient: with e = exp(-|a|), s = 1 / (1 + exp(-a)),
//   of a: grad_y * b * s * (1 + a * (1 - s)),  of b: grad_y * a * s.
// A thread has eight (fp32: four) neighbouring features of a row.  Bound by memory.
// ---------------------------------------------------------------------------
struct GateGradArgs {
  const void *grad_y, *sums;
  void* grad_sums;
  const int32_t* offset;
  int rows, slots, features;
};

__device__ __forceinline__ int clamp_row(int o, int rows) { return o < 0 ? 0 : o > rows ? rows : o; }

__device__ __forceinline__ void gate_grad(float grad, float a, float b, float* of_a, float* of_b) {
  const float e = expf(-fabsf(a)), below = 1.0f / (1.0f + e);
  const float s = a < 0.0f ? e * below : below, rest = a < 0.0f ? below : e * below;
  *of_a = grad * b * (s * fmaf(a, rest, 1.0f));
  *of_b = grad * (a * s);
}

template <bool BF16>
__global__ __launch_bounds__(256) void k_gate_grad(GateGradArgs a, int64_t first_piece) {
  constexpr int N = BF16 ? 8 : 4;
  const int64_t pieces = a.features / N, piece = first_piece + (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = piece / pieces, v = piece - row * pieces;
  int lo = 0, hi = a.rows;
  if (a.offset != nullptr) {
    lo = clamp_row(a.offset[0], a.rows);
    hi = clamp_row(a.offset[a.slots], a.rows);
  }
  if (row < lo || row >= hi) return;
  const u32x4 g = __builtin_nontemporal_load((const u32x4*)a.grad_y + row * pieces + v);
  const u32x4 x = __builtin_nontemporal_load((const u32x4*)a.sums + row * 2 * pieces + v);
  const u32x4 y = __builtin_nontemporal_load((const u32x4*)a.sums + (row * 2 + 1) * pieces + v);
  u32x4 of_x, of_y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float p[2], q[2];
    if constexpr (BF16) {
      gate_grad(bf16_lo(g[i]), bf16_lo(x[i]), bf16_lo(y[i]), &p[0], &q[0]);
      gate_grad(bf16_hi(g[i]), bf16_hi(x[i]), bf16_hi(y[i]), &p[1], &q[1]);
      of_x[i] = pack_bf16x2(p[0], p[1]);
      of_y[i] = pack_bf16x2(q[0], q[1]);
    } else {
      gate_grad(__uint_as_float(g[i]), __uint_as_float(x[i]), __uint_as_float(y[i]), &p[0], &q[0]);
      of_x[i] = __float_as_uint(p[0]);
      of_y[i] = __float_as_uint(q[0]);
    }
  }
  ((u32x4*)a.grad_sums)[row * 2 * pieces + v] = of_x;
  ((u32x4*)a.grad_sums)[(row * 2 + 1) * pieces + v] = of_y;
}

// ---------------------------------------------------------------------------
// tiles: 256 in_features by 64 * TT rows of the result, which are tokens (OF_W false: the rows' gradient, summed over the
// weights' rows) or weight rows (OF_W: the weights' gradient, summed over a slot's tokens).
//
// As in product.hip the in_features are the matrix cores' rows, so that a lane has four neighbouring ones of one row of the
// result.  Eight wavefronts; every step's operands come through LDS by direct loads, a step ahead, past the end of a tile into the
// next one's first step.
// ---------------------------------------------------------------------------
struct TileArgs {
  const uint8_t *g, *other;  // g: of the sums; other: the weights, or the rows x
  const int32_t* offset;
  uint8_t* out;
  int rows, slots;
  int n, k;           // weight rows (features of g), in_features
  int feature_tiles;  // of in_features
  int row_tiles;      // OF_W: of weight rows
  int64_t stride;     // bytes, from one slot's weights (or gradients) to the next one's
  int accumulate;
};

constexpr int kGradWaves = 8, kGradCols = 256;
constexpr int grad_across(int tt) { return tt == 4 ? 2 : 4; }  // wavefronts side by side on the columns
constexpr int grad_lds_bytes(int tt) { return 2 * (kGradCols + 64 * tt) * kStepBytes; }

// An operand that lies across the sum: rows of COLS values, in LDS one behind the other.  Its 16-byte chunks change places within a
// row, by a number that differs between the rows that are read at a time, so that these do not meet in the banks.
template <int DT, int COLS>
struct Across {
  static constexpr int kSize = DT == EEP_BF16 ? 2 : 4, kDepth = kStepBytes / kSize;
  static constexpr int kRowBytes = COLS * kSize, kChunks = kRowBytes / 16;
  static constexpr int kLoads = kDepth * kRowBytes / 1024 / kGradWaves;  // a wavefront's, of 1 KiB
  static_assert(kChunks >= 16 && kLoads >= 1, "");
  __device__ __forceinline__ static int places(int row) {
    return DT == EEP_BF16 ? 2 * ((row & 3) | ((row >> 1) & 4)) : 4 * ((row >> 2) & 3);
  }
  // The row and the first column that this lane brings in the i-th load.
  __device__ __forceinline__ static int row(int wave, int lane, int i) {
    return ((wave * kLoads + i) * 64 + lane) / kChunks;
  }
  __device__ __forceinline__ static int column(int wave, int lane, int i) {
    return ((lane % kChunks) ^ places(row(wave, lane, i))) * (16 / kSize);
  }
  // 16 columns from `tile` * 16 on.
  __device__ __forceinline__ static Frag read(const uint8_t* lds, int lane, int tile) {
    const int part = lane >> 4;
    Frag f;
    if constexpr (DT == EEP_BF16) {
      typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) i16x4 lds_quad;
      const int row = 8 * part + ((lane >> 2) & 3);
      const uint8_t* from = lds + row * kRowBytes + (((2 * tile + ((lane >> 1) & 1)) ^ places(row)) << 4) + (lane & 1) * 8;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x2 d = __builtin_bit_cast(
              u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad*)(from + (32 * j + 4 * h) * kRowBytes)));
          f.c[j][2 * h] = d[0];
          f.c[j][2 * h + 1] = d[1];
        }
    } else {
      const uint8_t* from =
          lds + 4 * part * kRowBytes + (((4 * tile + ((lane >> 2) & 3)) ^ places(4 * part)) << 4) + (lane & 3) * 4;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) f.c[j][i] = *(const uint32_t*)(from + (16 * j + i) * kRowBytes);
    }
    return f;
  }
};

// 16 bytes a lane from `offset` behind base, into LDS: the lanes' one behind the other.  The compiler, which cannot tell the turning
// reads of one stage from the loads into another, waits for its own loads of this kind before every such read; it does not know of
// these, and the kernel waits for them itself.  (The distance is that between a vector instruction that wrote a scalar register
// and the load that reads it, which is not kept for asm either.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 on the clobber list: nothing else here uses it)
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t offset, uint8_t* to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)to);
  const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
  const uint32_t high = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32));
  const uint64_t from = (uint64_t)high << 32 | low;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// Zeros in the place of the terms from `left` on.
template <int DT>
__device__ __forceinline__ void cut(Frag& f, int part, int left) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == EEP_BF16) {
        const int term = 32 * j + 8 * part + 2 * i;
        f.c[j][i] &= term + 1 < left ? 0xffffffffu : term < left ? 0xffffu : 0u;
      } else {
        f.c[j][i] = 16 * j + 4 * part + i < left ? f.c[j][i] : 0u;
      }
    }
}

template <int DT, int OT, bool OF_W, int TT>
__global__ __launch_bounds__(64 * kGradWaves, 2) void k_grad_tiled(TileArgs a) {
  constexpr int kWM = grad_across(TT), kWN = kGradWaves / kWM;
  constexpr int kA = kGradCols / 16 / kWM, kB = 4 * TT / kWN;  // tiles of 16 columns and of 16 rows a wavefront
  constexpr int kRows = 64 * TT;
  typedef Across<DT, kGradCols> Other;
  typedef Across<DT, OF_W ? kRows : kGradCols> Grads;  // (where they lie across too)
  constexpr int kSize = Other::kSize, kDepth = Other::kDepth;
  constexpr int kOtherStage = kGradCols * kStepBytes, kStage = kOtherStage + kRows * kStepBytes;
  constexpr int kLoads = kRows / 8 / kGradWaves;  // of g where its rows lie along the sum: 8 rows each
  extern __shared__ __align__(1024) uint8_t lds[];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % kWM, wn = wave / kWM;
  const int col = lane & 15, part = lane >> 4;

  struct Tile {
    int slot, column0, row0, first, end, steps;  // row0: of the result; first, end: the slot's rows (OF_W) or the tile's
  };
  TileMap<kRows> map;
  int64_t items, per_slot = 0;
  if constexpr (OF_W) {
    per_slot = (int64_t)a.row_tiles * a.feature_tiles;
    items = per_slot * a.slots;
  } else {
    map.make(a);
    items = (int64_t)map.total * a.feature_tiles;
  }
  // The items go to the XCDs in turn, 32 neighbouring ones at a time (as many as one has CUs), which share rows of the
  // operands in its L2.
  const int xcds = gridDim.x % 8 == 0 ? 8 : 1;
  const int xcd = blockIdx.x % xcds, seat = blockIdx.x / xcds, seats = gridDim.x / xcds;
  const auto item_of = [&](int64_t turn) { return turn / seats * seats * xcds + (int64_t)xcd * seats + turn % seats; };
  const auto find = [&](int64_t item) {
    Tile t;
    if constexpr (OF_W) {
      t.slot = (int)(item / per_slot);
      int at = (int)(item - t.slot * per_slot);
      // four tiles of weight rows by all of in_features, then the next four
      const int four = at / (4 * a.feature_tiles), tall = a.row_tiles - 4 * four < 4 ? a.row_tiles - 4 * four : 4;
      at -= four * 4 * a.feature_tiles;
      t.column0 = at / tall * kGradCols;
      t.row0 = (4 * four + at % tall) * kRows;
      t.first = 0;
      t.end = a.rows;
      if (a.offset != nullptr) {
        t.first = clamp_row(a.offset[t.slot], a.rows);
        t.end = clamp_row(a.offset[t.slot + 1], a.rows);
      }
      t.steps = t.end > t.first ? (t.end - t.first + kDepth - 1) / kDepth : 0;
    } else {
      int feature_tile;
      map.find(a, item, &t.slot, &feature_tile, &t.first, &t.end);
      t.column0 = feature_tile * kGradCols;
      t.row0 = t.first;
      t.steps = (a.n + kDepth - 1) / kDepth;
    }
    return t;
  };

  const int64_t k_bytes = (int64_t)a.k * kSize, n_bytes = (int64_t)a.n * kSize;
  // what the lane loads of g where its rows lie along the sum: 16 bytes of row `lane / 8` of eight
  const int load_row = lane >> 3, load_chunk = (lane & 7) ^ load_row;
  const auto fetch = [&](const Tile& t, int step, uint8_t* stage) {
    const int64_t at = (int64_t)step * kDepth;
    // terms past the end are read as the last ones, and cut off in the registers; columns likewise, and not stored
    const int left = (int)((OF_W ? t.end - t.first : a.n) - at);
    const uint8_t* other = OF_W ? a.other + (t.first + at) * k_bytes : a.other + t.slot * a.stride + at * k_bytes;
#pragma unroll
    for (int i = 0; i < Other::kLoads; ++i) {
      int r = Other::row(wave, lane, i), c = t.column0 + Other::column(wave, lane, i);
      r = r < left ? r : left - 1;
      c = c < a.k ? c : a.k - 16 / kSize;
      load_to_lds(other, (uint32_t)r * (uint32_t)k_bytes + (uint32_t)c * kSize, stage + (wave * Other::kLoads + i) * 1024);
    }
    if constexpr (OF_W) {
      const uint8_t* grads = a.g + (t.first + at) * n_bytes;
#pragma unroll
      for (int i = 0; i < Grads::kLoads; ++i) {
        int r = Grads::row(wave, lane, i), c = t.row0 + Grads::column(wave, lane, i);
        r = r < left ? r : left - 1;
        c = c < a.n ? c : a.n - 16 / kSize;
        load_to_lds(grads, (uint32_t)r * (uint32_t)n_bytes + (uint32_t)c * kSize,
                    stage + kOtherStage + (wave * Grads::kLoads + i) * 1024);
      }
    } else {
      const uint8_t* grads = a.g + t.first * n_bytes + at * kSize;
      const int chunk = load_chunk * (16 / kSize) < left ? load_chunk : 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        // (eight rows at a time are within 32 bits, all of them may not be)
        const int r0 = (wave * kLoads + i) * 8, most = t.end - 1 - t.first;
        const int from = r0 < most ? r0 : most, r = r0 + load_row < most ? r0 + load_row : most;
        load_to_lds(grads + from * n_bytes, (uint32_t)(r - from) * (uint32_t)n_bytes + chunk * 16,
                    stage + kOtherStage + (wave * kLoads + i) * 1024);
      }
    }
  };
  const int read_at = col * kStepBytes + ((part ^ (col & 7)) << 4);
  const auto read_other = [&](const uint8_t* stage, int f) { return Other::read(stage, lane, wm * kA + f); };
  const auto read_grads = [&](const uint8_t* stage, int j) {
    if constexpr (OF_W) {
      return Grads::read(stage + kOtherStage, lane, wn * kB + j);
    } else {
      Frag f;
      const uint8_t* from = stage + kOtherStage + (wn * kB + j) * 16 * kStepBytes;
      f.c[0] = *(const u32x4*)(from + read_at);
      f.c[1] = *(const u32x4*)(from + (read_at ^ 64));
      return f;
    }
  };

  int64_t turn = seat;
  int64_t item = item_of(turn);
  if (item >= items) return;
  Tile t = find(item);
  uint8_t *stage = lds, *following = lds + kStage;
  bool fetched = false;
  for (;;) {
    if (!fetched && t.steps > 0) fetch(t, 0, stage);
    fetched = false;
    const int64_t next_item = item_of(turn + seats);
    const bool more = next_item < items;
    Tile next = t;
    if (more) next = find(next_item);
    f32x4 acc[kA][kB];
#pragma unroll
    for (int f = 0; f < kA; ++f)
#pragma unroll
      for (int j = 0; j < kB; ++j) acc[f][j] = f32x4{0, 0, 0, 0};
    const int whole = OF_W ? (t.end > t.first ? (t.end - t.first) / kDepth : 0) : a.n / kDepth;
    const int left = OF_W ? t.end - t.first - whole * kDepth : a.n - whole * kDepth;
    const auto step = [&](int s, auto is_cut) {
      // This step's rows are there, and all wavefronts are done with the step before, whose place the next ones take.
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (s + 1 < t.steps) {
        fetch(t, s + 1, following);
      } else if (more && next.steps > 0) {
        fetch(next, 0, following);
        fetched = true;
      }
      Frag b[kB];
#pragma unroll
      for (int j = 0; j < kB; ++j) {
        b[j] = read_grads(stage, j);
        if constexpr (decltype(is_cut)::value) cut<DT>(b[j], part, left);
      }
#pragma unroll
      for (int f = 0; f < kA; ++f) {
        Frag v = read_other(stage, f);
        if constexpr (decltype(is_cut)::value) cut<DT>(v, part, left);
#pragma unroll
        for (int j = 0; j < kB; ++j) acc[f][j] = mma<DT>(v, b[j], acc[f][j]);
      }
      uint8_t* other = stage;
      stage = following;
      following = other;
    };
    for (int s = 0; s < whole; ++s) step(s, std::false_type());
    if (t.steps > whole) step(whole, std::true_type());

    const int rows_end = OF_W ? a.n : t.end;
    uint8_t* out = OF_W ? a.out + t.slot * a.stride : a.out;
    const int n0 = t.column0 + wm * (kA * 16);
#pragma unroll
    for (int j = 0; j < kB; ++j) {
      const int64_t row = (int64_t)t.row0 + (wn * kB + j) * 16 + col;
      const bool in = row < rows_end;
      if constexpr (OF_W) {
        if (a.accumulate != 0) {
          if (t.steps == 0) continue;  // (nothing to add)
#pragma unroll
          for (int f = 0; f < kA; ++f) {
            const int n = n0 + f * 16 + part * 4;
            if (!in || n >= a.k) continue;
            if constexpr (OT == EEP_F32) {
              acc[f][j] += *(const f32x4*)(out + (row * a.k + n) * 4);
            } else {
              const u32x2 d = *(const u32x2*)(out + (row * a.k + n) * 2);
              acc[f][j] += f32x4{bf16_lo(d[0]), bf16_hi(d[0]), bf16_lo(d[1]), bf16_hi(d[1])};
            }
          }
        }
      }
      if constexpr (OT == EEP_BF16) {
#pragma unroll
        for (int f = 0; f < kA; f += 2) store_tiles(out, row, a.k, n0 + f * 16, part, in, acc[f][j], acc[f + 1][j]);
      } else {
#pragma unroll
        for (int f = 0; f < kA; ++f) {
          const int n = n0 + f * 16 + part * 4;
          const float v[4] = {acc[f][j][0], acc[f][j][1], acc[f][j][2], acc[f][j][3]};
          if (in && n < a.k) store4<OT>(out, row * a.k + n, v);
        }
      }
    }
    if (!more) break;
    turn += seats;
    item = next_item;
    t = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may still write to LDS when the workgroup is gone
}

template <int DT, int OT, bool OF_W, int TT>
static hipError_t launch_grad_tiled(const TileArgs& a, int64_t work, int cus, hipStream_t st) {
  hipLaunchKernelGGL((k_grad_tiled<DT, OT, OF_W, TT>), dim3((unsigned)(work < cus ? work : cus)), dim3(64 * kGradWaves),
                     grad_lds_bytes(TT), st, a);
  return hipGetLastError();
}

template <int DT>
static hipError_t launch_grad_x(TileArgs a, int cus, hipStream_t st) {
  a.feature_tiles = (a.k + kGradCols - 1) / kGradCols;
  const int64_t touched = a.rows < a.slots ? a.rows : a.slots;
  const auto work = [&](int tokens) { return (a.rows + touched * (tokens - 1)) / tokens * a.feature_tiles; };
  const int mean = (int)((a.rows + a.slots - 1) / a.slots);
  if (mean <= 64) return launch_grad_tiled<DT, DT, false, 1>(a, work(64), cus, st);
  if (mean <= 128) return launch_grad_tiled<DT, DT, false, 2>(a, work(128), cus, st);
  return launch_grad_tiled<DT, DT, false, 4>(a, work(256), cus, st);
}

template <int DT, int OT>
static hipError_t launch_grad_w(TileArgs a, int cus, hipStream_t st) {
  a.feature_tiles = (a.k + kGradCols - 1) / kGradCols;
  const auto tiled = [&](auto tt) {
    constexpr int TT = decltype(tt)::value;
    a.row_tiles = (a.n + 64 * TT - 1) / (64 * TT);
    return launch_grad_tiled<DT, OT, true, TT>(a, (int64_t)a.row_tiles * a.feature_tiles * a.slots, cus, st);
  };
  return tiled(std::integral_constant<int, 4>());
}

// More LDS than a kernel may have by default, on the current device.
template <int DT>
static hipError_t allow_grad_lds() {
  const auto allow = [](const void* kernel, int tt) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, grad_lds_bytes(tt));
  };
  hipError_t e = allow((const void*)k_grad_tiled<DT, DT, false, 1>, 1);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, DT, false, 2>, 2);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, DT, false, 4>, 4);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, true, 4>, 4);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_BF16, true, 4>, 4);
  return e;
}

static bool overlaps(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  return a != nullptr && b != nullptr && (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

}  // namespace eep

using namespace eep;

extern "C" {

int eep_product_grad_create(const eep_product_grad_config* cfg, eep_product_grad** out) {
  if (!out) return EEP_ERR_INVALID_ARG;
  *out = nullptr;
  if (!cfg) return EEP_ERR_INVALID_ARG;
  const eep_product_grad_config& f = *cfg;
  const bool gated = f.gate == EEP_GATE_SILU;
  if (f.num_slots < 1 || f.num_slots > 65536 || f.in_features < 1 || f.out_features < 1 || f.in_features > (1 << 21) ||
      f.out_features > (1 << 21) || f.max_rows < 0 || f.max_rows > (1 << 30) || !f32_or_bf16(f.dtype) ||
      !f32_or_bf16(f.grad_w_dtype) || (!gated && f.gate != EEP_GATE_NONE))
    return EEP_ERR_INVALID_ARG;
  const int64_t in_bytes = (int64_t)f.in_features * dtype_bytes(f.dtype);
  const int64_t grad_row = (int64_t)f.in_features * dtype_bytes(f.grad_w_dtype);
  if (in_bytes % 16 || grad_row % 16 || (int64_t)f.out_features * dtype_bytes(f.dtype) % 16) return EEP_ERR_ALIGN;
  const int64_t weight_rows = (int64_t)f.out_features * (gated ? 2 : 1);
  if (f.slot_stride < 0 || f.grad_stride < 0 || (f.slot_stride != 0 && f.slot_stride < weight_rows * in_bytes) ||
      (f.grad_stride != 0 && f.grad_stride < weight_rows * grad_row))
    return EEP_ERR_INVALID_ARG;
  if (f.slot_stride % 16 || f.grad_stride % 16) return EEP_ERR_ALIGN;
  eep_product_grad* g = new (std::nothrow) eep_product_grad();
  if (!g) return EEP_ERR_INVALID_ARG;
  g->cfg = f;
  g->slot_stride = f.slot_stride ? f.slot_stride : weight_rows * in_bytes;
  g->grad_stride = f.grad_stride ? f.grad_stride : weight_rows * grad_row;
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess ||
      hipDeviceGetAttribute(&g->cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess ||
      (f.dtype == EEP_BF16 ? allow_grad_lds<EEP_BF16>() : allow_grad_lds<EEP_F32>()) != hipSuccess) {
    (void)hipGetLastError();
    delete g;
    return EEP_ERR_HIP;
  }
  *out = g;
  return EEP_OK;
}

int eep_product_grad_destroy(eep_product_grad* grad) {
  if (!grad) return EEP_OK;
  const hipError_t e = hipDeviceSynchronize();
  delete grad;
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

int eep_product_grad_run(eep_product_grad* grad, const void* grad_y, const void* sums, const void* x, const void* w,
                         const int32_t* offset, void* grad_sums, void* grad_x, void* grad_w, int32_t accumulate, int32_t rows,
                         void* stream) {
  if (!grad || rows < 0 || rows > grad->cfg.max_rows || (accumulate != 0 && accumulate != 1)) return EEP_ERR_INVALID_ARG;
  const eep_product_grad_config& f = grad->cfg;
  const bool gated = f.gate == EEP_GATE_SILU;
  if ((!gated && (sums || grad_sums)) || (!gated && !grad_x && !grad_w) || (gated && !grad_sums) || (offset == nullptr && f.num_slots != 1))
    return EEP_ERR_INVALID_ARG;
  if (rows > 0 && (!grad_y || (gated && !sums) || (grad_x && !w) || (grad_w && !x))) return EEP_ERR_INVALID_ARG;
  for (const void* p : {grad_y, sums, x, w, (const void*)grad_sums, (const void*)grad_x, (const void*)grad_w})
    if (!aligned16(p)) return EEP_ERR_ALIGN;
  if ((uintptr_t)offset & 3u) return EEP_ERR_ALIGN;
  const int size = dtype_bytes(f.dtype), n = f.out_features * (gated ? 2 : 1);
  const int64_t x_bytes = (int64_t)rows * f.in_features * size, y_bytes = (int64_t)rows * f.out_features * size;
  const int64_t sums_bytes = gated ? 2 * y_bytes : 0;
  const int64_t w_bytes = (f.num_slots - 1) * grad->slot_stride + (int64_t)n * f.in_features * size;
  const int64_t grad_w_bytes = (f.num_slots - 1) * grad->grad_stride + (int64_t)n * f.in_features * dtype_bytes(f.grad_w_dtype);
  const struct {
    const void* at;
    int64_t bytes;
  } from[] = {{grad_y, y_bytes}, {sums, sums_bytes}, {x, x_bytes}, {w, w_bytes}},
    to[] = {{grad_sums, sums_bytes}, {grad_x, x_bytes}, {grad_w, grad_w_bytes}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& o : from)
      if (overlaps(to[i].at, to[i].bytes, o.at, o.bytes) && !(i == 0 && o.at == sums && sums == grad_sums)) return EEP_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlaps(to[i].at, to[i].bytes, to[j].at, to[j].bytes)) return EEP_ERR_INVALID_ARG;
  }
  hipStream_t st = (hipStream_t)stream;
  const bool bf16 = f.dtype == EEP_BF16;
  hipError_t e = hipSuccess;
  if (gated && rows > 0) {
    const GateGradArgs a = {grad_y, sums, grad_sums, offset, rows, f.num_slots, f.out_features};
    const int64_t pieces = (int64_t)rows * (f.out_features / (bf16 ? 8 : 4));
    e = in_launches(pieces, max_blocks(256) * 256, [&](int64_t first, int64_t count) {
      hipLaunchKernelGGL((bf16 ? k_gate_grad<true> : k_gate_grad<false>), dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, a,
                         first);
      return hipGetLastError();
    });
  }
  TileArgs a = {};
  a.g = (const uint8_t*)(gated ? grad_sums : grad_y);
  a.offset = offset;
  a.rows = rows;
  a.slots = f.num_slots;
  a.n = n;
  a.k = f.in_features;
  a.accumulate = accumulate;
  if (e == hipSuccess && grad_x && rows > 0) {
    a.other = (const uint8_t*)w;
    a.out = (uint8_t*)grad_x;
    a.stride = grad->slot_stride;
    e = bf16 ? launch_grad_x<EEP_BF16>(a, grad->cus, st) : launch_grad_x<EEP_F32>(a, grad->cus, st);
  }
  if (e == hipSuccess && grad_w) {
    a.other = (const uint8_t*)x;
    a.out = (uint8_t*)grad_w;
    a.stride = grad->grad_stride;
    const bool out16 = f.grad_w_dtype == EEP_BF16;
    e = bf16 ? (out16 ? launch_grad_w<EEP_BF16, EEP_BF16>(a, grad->cus, st) : launch_grad_w<EEP_BF16, EEP_F32>(a, grad->cus, st))
             : (out16 ? launch_grad_w<EEP_F32, EEP_BF16>(a, grad->cus, st) : launch_grad_w<EEP_F32, EEP_F32>(a, grad->cus, st));
  }
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

}  // extern "C"
