// The gradients of the experts' products: of the rows, of every slot's weights, and of the gate between.
//
// Both products have an operand whose rows lie across the sum: the weights, whose in_features are neighbours while the sum goes
// over their rows; and for the weights' gradient both, since that sum goes over tokens.  Such an operand goes through LDS as it lies in
// memory, a step of 64 bytes' worth of the sum deep, and is turned on the way to the registers: ds_read_b64_tr_b16 gives a lane four
// values of ONE column from four rows (fp32 values are read one by one).  Lane l then has row (column) l % 16 and the 16 bytes' worth of
// terms from 16 * (l / 16) bytes into the step on.
#include <math.h>

#include <new>
#include <type_traits>

#include "eep_internal.hpp"
#include "numbers.hpp"
#include "tiles.hpp"

struct eep_product_grad {
  eep_product_grad_config cfg;
  int64_t slot_stride, grad_stride;  // bytes
  int cus;                           // of the device
  float* partial;                    // kPartialBytes of sums over parts of the terms
};

namespace eep {

// ---------------------------------------------------------------------------
// the gate's gradient: with e = exp(-|a|), s = 1 / (1 + exp(-a)),
//   of a: grad_y * b * s * (1 + a * (1 - s)),  of b: grad_y * a * s.
// A thread has eight (fp32: four) neighbouring features of a row.  Bound by memory: 131072 rows of 2 x 2048 bf16 429 us (6.3 TB/s).
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
// tiles: 256 in_features by 64 * TT rows (TT 0: 16; OF_W has 4 and 1, fp32 no 4) of the result, which are tokens (OF_W false: the rows' gradient, summed
// over the weights' rows) or weight rows (OF_W: the weights' gradient, summed over a slot's tokens).
//
// The in_features are the matrix cores' columns: a lane has one of them in four rows of the result, and they are dealt out to the lanes so
// that after an exchange among every four lanes it has four neighbouring ones of a row, and the 16 lanes beside one another 64 of them.
// (A CU stores 64 bytes at a time of what four neighbouring lanes have: where these are on different rows, a tile of 256 KB takes 8.0 us, now 2.0.)
// Eight wavefronts, or two workgroups of four to a CU for 64 and 16 rows; the steps of all tiles are one stream, of which some are under way to LDS while one is
// multiplied, and the operands that a step begins with are read while the one before ends.
// A step is 64 bytes deep, half of what is common, since the next tile's first steps are to be under way beside the stores of the last one: four
// stages instead of two (with stores that the waits count, 64 tokens 522 -> 490 us); five, which just fit, change nothing.  A step of 256 x 256 takes 0.76 us on few CUs,
// 0.87 to 1.05 on all, where the card's power bounds it too (131072 rows 4096 x 4096 0.97 and 1.02 PFLOP/s on normal random numbers; torch's product of 8192 x 8192 1.13);
// where stores are as many as products, one waits for the other: 120 slots 2880 -> 2816 of 304 tokens, fp32 gradients, 16 us a tile, of which
// the stores alone are 12.
// ---------------------------------------------------------------------------
struct TileArgs {
  const uint8_t *g, *other;  // g: of the sums; other: the weights, or the rows x
  const int32_t* offset;
  uint8_t* out;
  int rows, slots;
  int n, k;           // weight rows (features of g), in_features
  int feature_tiles;  // of in_features
  int row_tiles;      // OF_W: of weight rows
  int64_t stride;     // bytes, from one slot's weights to the next one's
  int64_t out_stride; // OF_W: and of their gradients
  int64_t plane;      // bytes, from one part's results to the next one's, where the terms are divided between gridDim.y
  int accumulate;
};

constexpr int kGradCols = 256, kGradStep = 64;  // bytes along the sum
constexpr int kGradStages = 4;
constexpr int grad_rows(int tt) { return tt == 0 ? 16 : 64 * tt; }
constexpr int grad_waves(int tt) { return tt == 4 ? 8 : 4; }
constexpr int grad_across(int tt) { return tt == 4 ? 2 : 4; }  // wavefronts side by side on the columns
constexpr int grad_stage_bytes(int tt) { return (kGradCols + grad_rows(tt)) * kGradStep; }
constexpr int grad_lds_bytes(int tt) { return kGradStages * grad_stage_bytes(tt); }
constexpr int grad_per_cu(int tt) { return tt == 4 ? 1 : 2; }  // workgroups

// One step of 16 rows (columns): lane l has four dwords of row l % 16, terms from 16 * (l / 16) bytes on.
template <int DT>
__device__ __forceinline__ f32x4 mma_step(const u32x4& a, const u32x4& b, f32x4 acc) {
  if constexpr (DT == EEP_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
    return acc;
  }
}

// 16 bytes a lane from `offset` behind base, into LDS: the lanes' one behind the other.  The compiler, which cannot tell the turning
// reads of one stage from the loads into another, waits for its own loads of this kind before every such read; it does not know of
// these, and the kernel waits for them itself.  (The distance is that between a vector instruction that wrote a scalar register
// and the load that reads it, which is not kept for asm either.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 on the clobber list: nothing else here uses it)
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t offset, uint32_t to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane(to);
  const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
  const uint32_t high = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32));
  const uint64_t from = (uint64_t)high << 32 | low;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// 16 or 8 bytes a lane: one store, whatever the compiler makes of what is around it.  past: the caches, non-temporal, for lines that are
// written whole.  (Data of 16 bytes has to stay for a while.)
template <class V>
__device__ __forceinline__ void store_counted(uint8_t* to, V v, bool past) {
  if constexpr (sizeof(V) == 16) {
    if (past)
      asm volatile("global_store_dwordx4 %0, %1, off nt\n\ts_nop 1" ::"v"(to), "v"(v) : "memory");
    else
      asm volatile("global_store_dwordx4 %0, %1, off\n\ts_nop 1" ::"v"(to), "v"(v) : "memory");
  } else {
    if (past)
      asm volatile("global_store_dwordx2 %0, %1, off nt" ::"v"(to), "v"(v) : "memory");
    else
      asm volatile("global_store_dwordx2 %0, %1, off" ::"v"(to), "v"(v) : "memory");
  }
}

// Lane p of every four has a, b, c, d; afterwards it has those of them that lanes 0 to 3 have at place p.  Every lane of the wavefront is there.
// (Each of the eight instructions takes a lane's own value or another's; what another lane wrote is read two instructions later at the soonest.)
__device__ __forceinline__ u32x4 turn_quads(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  uint32_t v, w, x, y, t, u;
#define EEP_OTHERS(to, other, own, lanes) "v_cndmask_b32_dpp " to ", " other ", " own ", vcc quad_perm:" lanes " row_mask:0xf bank_mask:0xf\n\t"
  asm volatile("s_nop 1\n\ts_mov_b64 vcc, %10\n\t"  // even lanes
               EEP_OTHERS("%4", "%7", "%6", "[1,0,3,2]") EEP_OTHERS("%2", "%9", "%8", "[1,0,3,2]")
               "s_mov_b64 vcc, %11\n\t"  // odd ones
               EEP_OTHERS("%5", "%6", "%7", "[1,0,3,2]") EEP_OTHERS("%3", "%8", "%9", "[1,0,3,2]")
               "s_mov_b64 vcc, %12\n\t"  // the lower two of four
               EEP_OTHERS("%0", "%2", "%4", "[2,3,0,1]") EEP_OTHERS("%1", "%3", "%5", "[2,3,0,1]")
               "s_mov_b64 vcc, %13\n\t"  // the upper two
               EEP_OTHERS("%2", "%4", "%2", "[2,3,0,1]") EEP_OTHERS("%3", "%5", "%3", "[2,3,0,1]")
               : "=&v"(v), "=&v"(w), "=&v"(x), "=&v"(y), "=&v"(t), "=&v"(u)
               : "v"(a), "v"(b), "v"(c), "v"(d), "s"(0x5555555555555555ull), "s"(0xaaaaaaaaaaaaaaaaull), "s"(0x3333333333333333ull),
                 "s"(0xccccccccccccccccull)
               : "vcc");
#undef EEP_OTHERS
  return u32x4{v, w, x, y};
}

// An operand that lies across the sum: rows of COLS values, in LDS one behind the other.  Its 16-byte chunks change places within a
// row, by a number that differs between the rows that are read at a time, so that these do not meet in the banks.
template <int DT, int COLS, int WAVES>
struct Across {
  static constexpr int kSize = DT == EEP_BF16 ? 2 : 4, kDepth = kGradStep / kSize;
  static constexpr int kRowBytes = COLS * kSize, kChunks = kRowBytes / 16;
  static constexpr int kLoads = kDepth * kRowBytes / 1024 / WAVES;  // a wavefront's, of 1 KiB
  static_assert(kChunks >= 8 && kLoads >= 1, "");
  __device__ __forceinline__ static int places(int row) {
    if constexpr (kChunks == 8)  // (of which two rows make one of all banks)
      return 2 * (((row >> 1) & 1) | ((row >> 2) & 2));
    else
      return DT == EEP_BF16 ? 2 * ((row & 3) | ((row >> 1) & 4)) : 4 * ((row >> 2) & 3);
  }
  // The row and the first column that this lane brings in the i-th load.
  __device__ __forceinline__ static int row(int wave, int lane, int i) {
    return ((wave * kLoads + i) * 64 + lane) / kChunks;
  }
  __device__ __forceinline__ static int column(int wave, int lane, int i) {
    return ((lane % kChunks) ^ places(row(wave, lane, i))) * (16 / kSize);
  }
  // Four neighbouring columns, counted in fours: those of lanes 4c to 4c + 3 of every 16 for the tile-th 16 columns.  spread: the columns of
  // four tiles change places, so that the lanes' values of the four make, after turn_quads, 64 neighbouring ones.
  template <bool SPREAD>
  __device__ __forceinline__ static int four(int c, int tile) {
    return SPREAD ? (tile >> 2) * 16 + c * 4 + ((tile & 3) ^ c) : tile * 4 + c;
  }
  // 16 columns of `tile`.
  template <bool SPREAD>
  __device__ __forceinline__ static u32x4 read(const uint8_t* lds, int lane, int tile) {
    const int part = lane >> 4;
    u32x4 f;
    if constexpr (DT == EEP_BF16) {
      typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) i16x4 lds_quad;
      const int row = 8 * part + ((lane >> 2) & 3), at = four<SPREAD>(lane & 3, tile);
      const uint8_t* from = lds + row * kRowBytes + (((at >> 1) ^ places(row)) << 4) + (at & 1) * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2 d =
            __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad*)(from + 4 * h * kRowBytes)));
        f[2 * h] = d[0];
        f[2 * h + 1] = d[1];
      }
    } else {
      const uint8_t* from =
          lds + 4 * part * kRowBytes + ((four<SPREAD>((lane >> 2) & 3, tile) ^ places(4 * part)) << 4) + (lane & 3) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = *(const uint32_t*)(from + i * kRowBytes);
    }
    return f;
  }
};

// Zeros in the place of the terms from `left` on.
template <int DT>
__device__ __forceinline__ void cut(u32x4& f, int part, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == EEP_BF16) {
      const int term = 8 * part + 2 * i;
      f[i] &= term + 1 < left ? 0xffffffffu : term < left ? 0xffffu : 0u;
    } else {
      f[i] = 4 * part + i < left ? f[i] : 0u;
    }
  }
}

template <int DT, int OT, bool OF_W, int TT>
__global__ __launch_bounds__(64 * grad_waves(TT), 2) void k_grad_tiled(TileArgs a) {
  constexpr int kWaves = grad_waves(TT), kWM = grad_across(TT), kWN = kWaves / kWM;
  constexpr int kRows = grad_rows(TT), kStages = kGradStages, kStage = grad_stage_bytes(TT);
  constexpr int kA = kGradCols / 16 / kWM, kB = kRows / 16 / kWN;  // tiles of 16 columns and of 16 rows a wavefront
  typedef Across<DT, kGradCols, kWaves> Other;
  typedef Across<DT, OF_W ? kRows : kGradCols, kWaves> Grads;  // (where they lie across too)
  constexpr int kSize = Other::kSize, kDepth = Other::kDepth;
  constexpr int kOtherStage = kGradCols * kGradStep;
  constexpr int kGradLoads = OF_W ? Grads::kLoads : TT == 0 ? 1 : kRows / 16 / kWaves;  // of g, a wavefront's; 16 rows each where they lie along
  constexpr int kLoads = Other::kLoads + kGradLoads;  // of a step
  extern __shared__ __align__(1024) uint8_t lds[];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % kWM, wn = wave / kWM;
  const int col = lane & 15, part = lane >> 4;

  struct Tile {
    int slot, column0, row0, first, end;  // row0: of the result; first, end: the slot's rows (OF_W) or the tile's
    int start, terms;                     // of the sum: this part's
  };
  const auto divide = [&](Tile& t) {
    t.start = 0;
    if (gridDim.y > 1) {
      const int64_t steps = (t.terms + kDepth - 1) / kDepth;
      const int end = (int)(steps * (blockIdx.y + 1) / gridDim.y) * kDepth;
      t.start = (int)(steps * blockIdx.y / gridDim.y) * kDepth;
      t.terms = (end < t.terms ? end : t.terms) - t.start;
    }
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
  // The items go to the XCDs in turn, as many neighbouring ones at a time as one has workgroups, which share rows of the
  // operands in its L2; what is left over for a last turn is divided between them.  Seats move on by one every turn: tiles of few rows
  // take less time, and come at even distances (120 slots 2880 -> 2816 of 300 tokens 1078 us with seats that stay, now 894; of 256 642 both).
  const int xcds = gridDim.x % 8 == 0 ? 8 : 1;
  const int xcd = blockIdx.x % xcds, seat = blockIdx.x / xcds, seats = gridDim.x / xcds;
  const int64_t whole_turns = items / gridDim.x, over = items - whole_turns * gridDim.x;
  const int over_from = (int)(over * xcd / xcds), over_to = (int)(over * (xcd + 1) / xcds);
  const int64_t turns = whole_turns + (seat < over_to - over_from ? 1 : 0);
  const auto item_of = [&](int64_t turn) {
    if (turn >= whole_turns) return turn * gridDim.x + over_from + seat;
    return turn * gridDim.x + xcd * seats + (int)(((unsigned)seat + (unsigned)turn) % (unsigned)seats);
  };
  // Where a walk over the items is: OF_W, the slot and the place among its tiles (without a division, which 64 bits make long).
  struct Walk {
    int64_t turn, at;
    int slot;
  };
  const auto find = [&](Walk& w) {
    Tile t;
    if constexpr (OF_W) {
      const int64_t item = item_of(w.turn);
      for (; item - w.at >= per_slot; w.at += per_slot) ++w.slot;
      t.slot = w.slot;
      int at = (int)(item - w.at);
      // four tiles of weight rows by all of in_features, then the next four
      const int four = at / (4 * a.feature_tiles), tall = a.row_tiles - 4 * four < 4 ? a.row_tiles - 4 * four : 4;
      at -= four * 4 * a.feature_tiles;
      t.column0 = at / tall * kGradCols;
      t.row0 = (4 * four + at % tall) * kRows;
      t.first = 0;
      t.end = a.rows;
      if (a.offset != nullptr) {
        // (scalar loads, for which nothing but themselves is awaited)
        const auto* offset = (const __attribute__((address_space(4))) int32_t*)a.offset;
        t.first = clamp_row(offset[t.slot], a.rows);
        t.end = clamp_row(offset[t.slot + 1], a.rows);
      }
      t.terms = t.end > t.first ? t.end - t.first : 0;
    } else {
      int feature_tile;
      map.find(a, item_of(w.turn), &t.slot, &feature_tile, &t.first, &t.end);
      t.column0 = feature_tile * kGradCols;
      t.row0 = t.first;
      t.terms = a.n;
    }
    divide(t);
    return t;
  };

  const int64_t k_bytes = (int64_t)a.k * kSize, n_bytes = (int64_t)a.n * kSize;
  // What the lane loads of g where its rows lie along the sum: 16 bytes of row `lane / 4` of 16.  A row's four chunks change places there so
  // that reads of 16 bytes meet in no bank: lanes 0 to 3, 12 to 15 and 20 to 27 take theirs at a time, 4 to 11, 16 to 19 and 28 to 31.
  const auto places = [](int row) {
    const int four = (row >> 2) & 3;
    return ((four & 1) << 1) ^ (four >> 1) ^ (four & 2);
  };
  const int load_row = lane >> 2, load_chunk = (lane & 3) ^ places(load_row);

  // The stream of steps: the tile that is fetched, its terms left, where its operands are and the lane's places there.
  Walk ahead = {-1, 0, 0};
  int fetch_left = 0;
  const uint8_t *other_at = nullptr, *grads_at[kGradLoads] = {};
  uint32_t other_off[Other::kLoads] = {}, grads_off[kGradLoads] = {};
  int stage_at = 0;  // of the next fetch
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_void*)lds;
  // (terms past the end are read as the last ones, and cut off in the registers; columns likewise, and not stored)
  const auto aim = [&](const Tile& t) {
    fetch_left = t.terms;
    other_at = (OF_W ? a.other + t.first * k_bytes : a.other + t.slot * a.stride) + t.start * k_bytes;
    other_at += (int64_t)t.column0 * kSize;
#pragma unroll
    for (int i = 0; i < Other::kLoads; ++i) {
      const int r = Other::row(wave, lane, i), c = Other::column(wave, lane, i), most = a.k - t.column0 - 16 / kSize;
      other_off[i] = (uint32_t)r * (uint32_t)k_bytes + (uint32_t)(c < most ? c : most) * kSize;
    }
    if constexpr (OF_W) {
#pragma unroll
      for (int i = 0; i < kGradLoads; ++i) {
        const int r = Grads::row(wave, lane, i), c = Grads::column(wave, lane, i), most = a.n - t.row0 - 16 / kSize;
        grads_at[i] = a.g + (t.first + t.start) * n_bytes + (int64_t)t.row0 * kSize;
        grads_off[i] = (uint32_t)r * (uint32_t)n_bytes + (uint32_t)(c < most ? c : most) * kSize;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kGradLoads; ++i) {
        // (16 rows at a time are within 32 bits, all of them may not be)
        const int r0 = TT == 0 ? 0 : (wave * kGradLoads + i) * 16, most = t.end > t.first ? t.end - 1 - t.first : 0;
        const int from = r0 < most ? r0 : most, r = r0 + load_row < most ? r0 + load_row : most;
        grads_at[i] = a.g + (t.first + from) * n_bytes + (int64_t)t.start * kSize;
        grads_off[i] = (uint32_t)(r - from) * (uint32_t)n_bytes + load_chunk * 16;
      }
    }
  };
  bool more = true;
  const auto fetch = [&]() {
    // (behind the stream's end nothing new: the last step again, so that as many loads are under way as ever)
    if (fetch_left <= 0 && more) {
      for (;;) {
        if (++ahead.turn >= turns) {
          more = false;
          break;
        }
        const Tile t = find(ahead);
        if (t.terms == 0) continue;
        aim(t);
        break;
      }
    }
    if (other_at == nullptr) return;  // (no tile has terms)
    const uint32_t to = lds_base + stage_at * kStage + wave * 1024;
    const bool again = !more && fetch_left <= 0;
    if (!again && fetch_left < kDepth) {
#pragma unroll
      for (int i = 0; i < Other::kLoads; ++i) {
        const int r = Other::row(wave, lane, i), last = fetch_left - 1;
        if (r > last) other_off[i] -= (uint32_t)(r - last) * (uint32_t)k_bytes;
      }
#pragma unroll
      for (int i = 0; i < kGradLoads; ++i) {
        if constexpr (OF_W) {
          const int r = Grads::row(wave, lane, i), last = fetch_left - 1;
          if (r > last) grads_off[i] -= (uint32_t)(r - last) * (uint32_t)n_bytes;
        } else if (load_chunk * (16 / kSize) >= fetch_left) {
          grads_off[i] -= load_chunk * 16;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < Other::kLoads; ++i) load_to_lds(other_at, other_off[i], to + wave * (Other::kLoads - 1) * 1024 + i * 1024);
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i)
      // (of 16 rows all wavefronts bring the same)
      load_to_lds(grads_at[i], grads_off[i], to + kOtherStage + (TT == 0 ? -wave * 1024 : wave * (kGradLoads - 1) * 1024 + i * 1024));
    stage_at = stage_at + 1 < kStages ? stage_at + 1 : 0;
    if (!again) {
      fetch_left -= kDepth;
      if (fetch_left > 0) {
        other_at += kDepth * k_bytes;
#pragma unroll
        for (int i = 0; i < kGradLoads; ++i) grads_at[i] += OF_W ? kDepth * n_bytes : kGradStep;
      }
    }
  };
  const int read_at = col * kGradStep + ((part ^ places(col)) << 4);
  // (a wavefront's four tiles at a time are 64 * kWM columns apart, which the places of chunks have no part in)
  const auto read_other = [&](const uint8_t* stage, int f) {
    return Other::template read<true>(stage + (f >> 2) * kWM * 64 * kSize, lane, wm * 4 + (f & 3));
  };
  const auto read_grads = [&](const uint8_t* stage, int j) {
    if constexpr (OF_W)
      return Grads::template read<false>(stage + kOtherStage, lane, wn * kB + j);
    else
      return *(const u32x4*)(stage + kOtherStage + (wn * kB + j) * 16 * kGradStep + read_at);
  };

  // the first tile that has terms at all
#pragma nounroll  // (its code comes three times as it is)
  for (int s = 0; s < kStages; ++s) fetch();
  const uint8_t* stage = lds;
  // What a step begins with: all of g's operands, the first ones of the other.
  constexpr int kAhead = 2, kBefore = kA - 2;
  static_assert(kBefore + kAhead >= kA, "all of the stage is read");
  u32x4 b_head[kB], a_head[kAhead];
  const auto read_heads = [&]() {
    a_head[0] = read_other(stage, 0);
#pragma unroll
    for (int j = 0; j < kB; ++j) b_head[j] = read_grads(stage, j);
#pragma unroll
    for (int f = 1; f < kAhead; ++f) a_head[f] = read_other(stage, f);
  };
  const bool any = other_at != nullptr;
  if (any) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_heads();
  }

  constexpr int kStores = kA * kB;  // of a whole tile, a wavefront's
  static_assert(kA % 4 == 0, "four tiles change places");
  static_assert((kStages - 2) * kLoads + kStores < 64, "what the counter holds");
  int behind_stores = kStages;  // steps since a whole tile was stored
  for (Walk here = {0, 0, 0}; here.turn < turns; ++here.turn) {
    const Tile t = find(here);
    const int rows_end = OF_W ? a.n : t.end;
    f32x4 acc[kA][kB];
#pragma unroll
    for (int f = 0; f < kA; ++f)
#pragma unroll
      for (int j = 0; j < kB; ++j) acc[f][j] = f32x4{0, 0, 0, 0};
    // All wavefronts have read what they need of the stage and the next step's rows are there (no more than the fetches behind them are
    // under way): the stage may be filled again and the next step's first operands are read.
    const auto turn_over = [&](bool heads) {
      // (Loads and stores count together, in order: the last tile's stores are newer than the rows of the next kStages - 1 steps.)
      if (behind_stores < kStages - 1)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * kLoads + kStores) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * kLoads) : "memory");
      ++behind_stores;
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      stage = stage + kStage < lds + kStages * kStage ? stage + kStage : lds;
      if (heads) read_heads();
      fetch();
    };
    const auto step = [&](int left, auto is_cut) {
      const auto ready = [&](u32x4 f) {
        if constexpr (decltype(is_cut)::value) cut<DT>(f, part, left);
        return f;
      };
      u32x4 b[kB], v[kA];
#pragma unroll
      for (int j = 0; j < kB; ++j) b[j] = ready(b_head[j]);
#pragma unroll
      for (int f = 0; f < kAhead; ++f) v[f] = a_head[f];
      const auto multiply = [&](int f) {
        const u32x4 now = ready(v[f]);
#pragma unroll
        for (int j = 0; j < kB; ++j) acc[f][j] = mma_step<DT>(b[j], now, acc[f][j]);
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int f = 0; f < kBefore; ++f) {
        if (f + kAhead < kA) v[f + kAhead] = read_other(stage, f + kAhead);
        multiply(f);
      }
      turn_over(true);
#pragma unroll
      for (int f = kBefore; f < kA; ++f) multiply(f);
    };
    // fp32 products, whose roundings show, are added up 512 terms at a time and these sums then: over 5632 terms 1.3e-6 off in the
    // 2-norm, now 0.4e-6.  (Tiles of 256 rows have no registers left for it, so fp32 has none: 5632 rows 5632 x 2432, both gradients, 2.78 ms
    // in such tiles, 2.95 in those of 64; tiles of 128, one to a CU, 3.03; of 43 other calls 0.82 to 1.12 of the time.)
    constexpr bool kFolds = DT == EEP_F32;
    static_assert(!kFolds || TT != 4, "two sets of sums");
    constexpr int kFoldSteps = 512 / kDepth;
    f32x4 total[kFolds ? kA : 1][kFolds ? kB : 1] = {};
    const auto fold_sums = [&](bool last) {
      if constexpr (kFolds) {
#pragma unroll
        for (int f = 0; f < kA; ++f)
#pragma unroll
          for (int j = 0; j < kB; ++j) {
            total[f][j] += acc[f][j];
            acc[f][j] = last ? total[f][j] : f32x4{0, 0, 0, 0};
          }
      }
    };
    int left = t.terms;
    if (OF_W || t.row0 + wn * kB * 16 < rows_end) {
      for (int steps = 1; left >= kDepth; left -= kDepth, ++steps) {
        step(left, std::false_type());
        if (kFolds && steps % kFoldSteps == 0) fold_sums(false);
      }
      if (left > 0) step(left, std::true_type());
      fold_sums(true);
    } else {
      // (none of this wavefront's rows is one: it only takes part in the fetches)
      for (; left > 0; left -= kDepth) turn_over(left <= kDepth);
    }

    uint8_t* out = a.out + blockIdx.y * a.plane + (OF_W ? t.slot * a.out_stride : 0);
    if (OF_W && a.accumulate != 0 && t.terms == 0) continue;  // (nothing to add)
    // The lane has, of rows row0 + 16 j + i, columns column + kNext * q to column + kNext * q + 3.
    constexpr int kOut = OT == EEP_F32 ? 4 : 2, kNext = 64 * kWM;
    const int column = t.column0 + wm * 64 + (col & 12) * 4 + (((col >> 2) ^ col) & 3) * 4;
    const int row0 = t.row0 + wn * kB * 16 + part * 4;
    // (the compiler, which keeps the matrix instructions' distance to what reads their results, does not look into turn_quads)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const auto values = [&](int j, int q, int i) {
      return turn_quads(__float_as_uint(acc[4 * q][j][i]), __float_as_uint(acc[4 * q + 1][j][i]), __float_as_uint(acc[4 * q + 2][j][i]),
                        __float_as_uint(acc[4 * q + 3][j][i]));
    };
    if (OF_W && a.accumulate != 0) {
#pragma unroll
      for (int j = 0; j < kB; ++j)
#pragma unroll
        for (int q = 0; q < kA / 4; ++q) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 v = __builtin_bit_cast(f32x4, values(j, q, i));
            const int row = row0 + j * 16 + i, n = column + q * kNext;
            if (row >= rows_end || n >= a.k) continue;
            uint8_t* to = out + ((int64_t)row * a.k + n) * kOut;
            if constexpr (OT == EEP_F32) {
              *(f32x4*)to = v + *(const f32x4*)to;
            } else {
              const u32x2 d = *(const u32x2*)to;
              *(u32x2*)to = u32x2{pack_bf16x2(v[0] + bf16_lo(d[0]), v[1] + bf16_hi(d[0])),
                                  pack_bf16x2(v[2] + bf16_lo(d[1]), v[3] + bf16_hi(d[1]))};
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      behind_stores = kStages;
      continue;
    }
    // A whole tile is stored by a number of stores that the steps behind them count on.
    const auto store = [&](auto is_whole) {
      constexpr bool kWhole = decltype(is_whole)::value;
      int64_t pitch = (int64_t)a.k * kOut;
      asm volatile("" : "+s"(pitch));  // (else all rows' distances are kept from tile to tile, in registers that are not there)
      uint8_t* to = out + row0 * pitch + (int64_t)column * kOut;
      const bool past = (((uintptr_t)out | (uint64_t)pitch) & 127u) == 0;
#pragma unroll
      for (int j = 0; j < kB; ++j)
#pragma unroll
        for (int q = 0; q < kA / 4; ++q) {
          const auto put = [&](int i, auto v) {
            if (kWhole || (row0 + j * 16 + i < rows_end && column + q * kNext < a.k))
              store_counted(to + ((j * 16 + i) * pitch + q * kNext * kOut), v, past);
          };
          if constexpr (OT == EEP_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) put(i, values(j, q, i));
          } else {
            // (two rows' values are turned together)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              uint32_t p[4];
#pragma unroll
              for (int f = 0; f < 4; ++f) p[f] = pack_bf16x2(acc[4 * q + f][j][i], acc[4 * q + f][j][i + 1]);
              const u32x4 v = turn_quads(p[0], p[1], p[2], p[3]);
              put(i, u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x05040100), __builtin_amdgcn_perm(v[3], v[2], 0x05040100)});
              put(i + 1, u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x07060302), __builtin_amdgcn_perm(v[3], v[2], 0x07060302)});
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (t.row0 + kRows <= rows_end && t.column0 + kGradCols <= a.k) {
      store(std::true_type());
      behind_stores = 0;
    } else {
      store(std::false_type());
      behind_stores = kStages;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may still write to LDS when the workgroup is gone
}

// The parts' sums, added in their order: of rows of `width` values, of which those of the slots alone (offset NULL: all).
struct PartArgs {
  const float* partial;
  const int32_t* offset;
  uint8_t* out;
  int64_t plane, slot_values, out_stride;  // values of a part and of a slot (0: one array), bytes from one slot's results to the next one's
  int width, rows, slots, parts, accumulate;
};
template <bool BF16>
__global__ __launch_bounds__(256) void k_grad_parts(PartArgs a) {
  int64_t from = 0, to = a.plane;
  if (a.offset != nullptr) {
    from = (int64_t)clamp_row(a.offset[0], a.rows) * a.width;
    to = (int64_t)clamp_row(a.offset[a.slots], a.rows) * a.width;
  }
  for (int64_t at = from + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; at < to; at += (int64_t)gridDim.x * 1024) {
    f32x4 sum = *(const f32x4*)(a.partial + at);
    int p = 1;
    for (; p + 8 <= a.parts; p += 8) {  // eight under way together
      f32x4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = *(const f32x4*)(a.partial + (p + i) * a.plane + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[i];
    }
    for (; p < a.parts; ++p) sum += *(const f32x4*)(a.partial + p * a.plane + at);
    const int64_t slot = a.slot_values != 0 ? at / a.slot_values : 0;
    uint8_t* to_slot = a.out + slot * a.out_stride;
    const int64_t in_slot = at - slot * a.slot_values;
    if constexpr (BF16) {
      u32x2* o = (u32x2*)to_slot + in_slot / 4;
      if (a.accumulate != 0) {
        const u32x2 d = *o;
        sum += f32x4{bf16_lo(d[0]), bf16_hi(d[0]), bf16_lo(d[1]), bf16_hi(d[1])};
      }
      *o = u32x2{pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    } else {
      f32x4* o = (f32x4*)to_slot + in_slot / 4;
      if (a.accumulate != 0) sum += *o;
      *o = sum;
    }
  }
}

// What a step of a tile takes, us: of 256 rows (bf16 alone has them); of 64 and 16, of which a CU has two, a step of both, or of one alone.  fp32 products take
// the matrix cores 16 times as long as bf16 ones, on half as many terms a step.
static float grad_step_time(int tt, bool f32, bool alone) {
  if (f32) return tt == 1 ? (alone ? 1.1f : 2.2f) : (alone ? 0.4f : 0.8f);
  return tt == 4 ? (alone ? 0.8f : 0.95f) : tt == 1 ? (alone ? 0.4f : 0.75f) : (alone ? 0.35f : 0.5f);
}

// Where tiles are few, the terms of each are divided between several workgroups, whose sums are left in the workspace and added up by a
// launch more: into as many parts as there are CUs for, of four steps at least (one, where it takes so long), unless writing and reading that many sums takes
// longer than the steps that it saves.  (664 rows 1720 x 1368: the weights' gradient in 5 parts 36 us, undivided 27; 249 rows 256 -> 1264 in
// fp32, both gradients, 47 us with four steps at least, 41 with one.)
constexpr int64_t kPartialBytes = 64 << 20;  // (256 CUs' tiles of 256 by 256)
static float grad_parts_time(int64_t parts, int64_t values) { return parts == 1 ? 0.0f : 6.0f + parts * values * 8 / 4.5e6f; }
static int grad_parts(int64_t work, int64_t most, int64_t steps, int64_t values, float step) {
  int64_t limit = work > 0 ? most / work : 1;
  const int64_t shortest = step > 1.0f ? 1 : 4;
  if (limit > steps / shortest) limit = steps / shortest;
  if (limit > kPartialBytes / (values * (int64_t)sizeof(float))) limit = kPartialBytes / (values * (int64_t)sizeof(float));
  if (limit < 2) return 1;
  const float best = sqrtf(step * steps / (values * 8 / 4.5e6f));
  const int64_t parts = best < limit ? (int64_t)best : limit;
  return parts >= 2 && step * steps / parts + grad_parts_time(parts, values) < step * steps ? (int)parts : 1;
}

// An fp32 step takes the matrix cores of a CU alike with one workgroup on it and with two: what counts is how many tiles the CU has that has
// most, so that 200 tiles on 256 CUs take as long as 256, and 300 as long as 512.  Divided into 2 to 8 parts they are spread more evenly, undivided / so,
// us: rows of 449 x 5760 -> 6400 392 / 329, weights 1024 x 5248 of 8311 rows with those rows' gradient 1884 / 1539, 9600 x 336 of 6620 1603 / 1295.
static float grad_time_f32(int64_t work, int64_t parts, int64_t steps, int64_t values, float step, int cus) {
  return (float)((work * parts + cus - 1) / cus) * step * steps / parts + grad_parts_time(parts, values);
}
static int grad_spread_f32(int64_t work, int parts, int64_t steps, int64_t values, float step, int cus) {
  const float now = grad_time_f32(work, parts, steps, values, step, cus);
  float least = 0.85f * now;  // (the tiles are an estimate)
  for (int p = 2; p <= 8 && p <= steps && p * values * (int64_t)sizeof(float) <= kPartialBytes; ++p) {
    const float time = grad_time_f32(work, p, steps, values, step, cus);
    if (time < least) {
      least = time;
      parts = p;
    }
  }
  return parts;
}

// values, width: of the result, of one of its rows; terms: of a sum, about.
template <int DT, int OT, bool OF_W, int TT>
static hipError_t launch_grad_tiled(const TileArgs& a, const eep_product_grad& g, int64_t work, int64_t values, int64_t terms,
                                    hipStream_t st) {
  constexpr int kDepth = kGradStep / (DT == EEP_BF16 ? 2 : 4);
  const int64_t most = (int64_t)g.cus * grad_per_cu(TT);
  const unsigned grid = (unsigned)(work < most ? work : most);
  const int64_t steps = (terms + kDepth - 1) / kDepth;
  const float step = grad_step_time(TT, DT == EEP_F32, true);
  int parts = grad_parts(work, most, steps, values, step);
  if (DT == EEP_F32) parts = grad_spread_f32(work, parts, steps, values, step, g.cus);
  if (parts == 1) {
    hipLaunchKernelGGL((k_grad_tiled<DT, OT, OF_W, TT>), dim3(grid), dim3(64 * grad_waves(TT)), grad_lds_bytes(TT), st, a);
    return hipGetLastError();
  }
  TileArgs part = a;
  part.out = (uint8_t*)g.partial;
  part.out_stride = (int64_t)a.n * a.k * (int64_t)sizeof(float);
  part.plane = values * (int64_t)sizeof(float);
  part.accumulate = 0;
  hipLaunchKernelGGL((k_grad_tiled<DT, EEP_F32, OF_W, TT>), dim3(grid, (unsigned)parts), dim3(64 * grad_waves(TT)), grad_lds_bytes(TT), st,
                     part);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const PartArgs sum = {g.partial, OF_W ? nullptr : a.offset, a.out, values, OF_W ? (int64_t)a.n * a.k : 0, a.out_stride, a.k,
                        a.rows, a.slots, parts, OF_W ? a.accumulate : 0};
  const int64_t blocks = (values / 4 + 255) / 256;
  hipLaunchKernelGGL((k_grad_parts<OT == EEP_BF16>), dim3((unsigned)(blocks < 4 * g.cus ? blocks : 4 * g.cus)), dim3(256), 0, st, sum);
  return hipGetLastError();
}

// What the tiles of 256, 64 or 16 tokens cost, us: their steps, as often as a CU has one, and the sum of parts.  A slot's last tile is half
// empty on average.  Measured, 16 / 64 / 256 tokens a tile, us, bf16: one matrix 256 x 7168, 64 tokens 9.6 / 11.2 / 15.2, 512 18.6 / 12.2 / 17.1, 4096
// 94 / 34.8 / 31.9; 2048 x 2048, 2048 tokens 68 / 37.9 / 49.5; 7168 x 2048, 512 64 / 37.4 / 44.4; eight slots 512 x 2048 of 1000 84 / 31.5 / 26.4; 120 slots
// 2816 x 2880 of 4 334 / 343 / 361, of 16 388 / 355 / 364, of 50 641 / 375 / 371, of 100 1000 / 530 / 418; fp32: 2048 x 2048, 2048 tokens 201 / 155, 120
// slots 2816 x 2880 of 4 686 / 1121.  (Tiles of 128 were between the two, and best nowhere.)
static float grad_x_cost(int tt, bool f32, const TileArgs& a, int64_t steps, int cus) {
  const int64_t touched = a.rows < a.slots ? a.rows : a.slots, most = (int64_t)cus * grad_per_cu(tt), rows = grad_rows(tt);
  float tiles = (float)a.rows / touched / rows + 0.5f;
  if (touched == 1) tiles = (float)((a.rows + rows - 1) / rows);
  const float work = (tiles < 1.0f ? 1.0f : tiles) * touched * a.feature_tiles;
  const int64_t values = (int64_t)a.rows * a.k;
  const float alone = grad_step_time(tt, f32, true);
  const int parts = grad_parts((int64_t)work, most, steps, values, alone);
  const float rounds = work * parts / most, step = grad_step_time(tt, f32, rounds <= 0.5f);
  float time = step * steps / parts * (rounds < 4.0f ? ceilf(rounds) : rounds) + grad_parts_time(parts, values);
  const int spread = f32 ? grad_spread_f32((int64_t)work, parts, steps, values, alone, cus) : parts;
  if (spread != parts) time = grad_time_f32((int64_t)work, spread, steps, values, alone, cus);
  // Weights that no cache holds come from memory for every tile of a slot, since its tiles are seldom at the same place; in tiles of 64 / 256,
  // us: 120 slots 2880 -> 2816 of 50 tokens 375 / 371, of 64 460 / 387, of 100 530 / 418, of 200 776 / 570; 144 slots 4096 -> 4096 of 50 858 / 785,
  // of 64 960 / 852, of 100 1111 / 914; 32 slots 7168 -> 2048 of 50 191 / 189, of 100 247 / 214; 144 slots 1024 -> 4096 of 50 238 / 263, of 100
  // 283 / 280.  Of 48 points of six shapes beside the first (16 to 200 tokens, 0.26 to 4.8 GB) what is chosen took 1.034 times the best of the three in the
  // mean, without this 1.065; either way 1.45 at most (16 slots 2880 -> 2816 of 80, 94 / 65).
  const float weights = (float)touched * a.n * a.k * (f32 ? 4 : 2), from_memory = (tiles < 1.0f ? 1.0f : tiles) * weights / 6.0e6f;
  if (weights > 256e6f) time = 0.05f * time + (time < from_memory ? from_memory : time);
  return time;
}

template <int DT>
static hipError_t launch_grad_x(TileArgs a, const eep_product_grad& g, hipStream_t st) {
  a.feature_tiles = (a.k + kGradCols - 1) / kGradCols;
  const int64_t touched = a.rows < a.slots ? a.rows : a.slots;
  const auto tiled = [&](auto tt) {
    constexpr int TT = decltype(tt)::value;
    return launch_grad_tiled<DT, DT, false, TT>(a, g, (a.rows + touched * (grad_rows(TT) - 1)) / grad_rows(TT) * a.feature_tiles,
                                                (int64_t)a.rows * a.k, a.n, st);
  };
  constexpr int kDepth = kGradStep / (DT == EEP_BF16 ? 2 : 4);
  const int sizes[] = {4, 1, 0};
  int best = 0;
  float least = INFINITY;
  for (const int tt : sizes) {
    if (DT == EEP_F32 && tt == 4) continue;
    const float cost = grad_x_cost(tt, DT == EEP_F32, a, (a.n + kDepth - 1) / kDepth, g.cus);
    if (cost < least) {
      least = cost;
      best = tt;
    }
  }
  if constexpr (DT != EEP_F32)
    if (best == 4) return tiled(std::integral_constant<int, 4>());
  return best == 1 ? tiled(std::integral_constant<int, 1>()) : tiled(std::integral_constant<int, 0>());
}

// The same for tiles of 256 or 64 weight rows, for bf16 (fp32 has but the latter).  Measured, 256 / 64, us: one matrix 256 x 7168, 64 rows 9.6 / 6.8, 512 20.2 / 13.0, 16384
// 89.8 / 98.1; 2048 x 2048, 2048 rows 44.7 / 35.1; 2048 x 7168, 128 rows 13.5 / 14.4; eight slots 512 x 2048 of 1000 rows 32.9 / 25.7, 1024 x 2048 of 300
// 19.0 / 21.5; 144 slots 4096 x 1024 of 4 rows 202 / 260.
static float grad_w_cost(int tt, const TileArgs& a, int64_t work, int64_t steps, int cus) {
  const int64_t most = (int64_t)cus * grad_per_cu(tt), values = (int64_t)a.slots * a.n * a.k;
  const float alone = grad_step_time(tt, false, true), both = grad_step_time(tt, false, false);
  const int parts = grad_parts(work, most, steps, values, alone);
  const float rounds = (float)work * parts / most, more = rounds < 0.5f ? 0.0f : rounds > 1.0f ? 1.0f : 2.0f * rounds - 1.0f;
  return (alone + (both - alone) * more) * steps / parts * (rounds < 4.0f ? ceilf(rounds) : rounds) + grad_parts_time(parts, values);
}

template <int DT, int OT>
static hipError_t launch_grad_w(TileArgs a, const eep_product_grad& g, hipStream_t st) {
  constexpr int kDepth = kGradStep / (DT == EEP_BF16 ? 2 : 4);
  a.feature_tiles = (a.k + kGradCols - 1) / kGradCols;
  const int64_t terms = a.rows / a.slots, steps = terms < kDepth ? 1 : (terms + kDepth - 1) / kDepth;
  const auto work = [&](int tt) { return (int64_t)((a.n + grad_rows(tt) - 1) / grad_rows(tt)) * a.feature_tiles * a.slots; };
  const auto tiled = [&](auto tt) {
    constexpr int TT = decltype(tt)::value;
    a.row_tiles = (a.n + grad_rows(TT) - 1) / grad_rows(TT);
    return launch_grad_tiled<DT, OT, true, TT>(a, g, work(TT), (int64_t)a.slots * a.n * a.k, terms, st);
  };
  if constexpr (DT != EEP_F32)
    if (!(grad_w_cost(1, a, work(1), steps, g.cus) < grad_w_cost(4, a, work(4), steps, g.cus)))
      return tiled(std::integral_constant<int, 4>());
  return tiled(std::integral_constant<int, 1>());
}

// More LDS than a kernel may have by default, on the current device.
template <int DT>
static hipError_t allow_grad_lds() {
  const auto allow = [](const void* kernel, int tt) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, grad_lds_bytes(tt));
  };
  hipError_t e = allow((const void*)k_grad_tiled<DT, DT, false, 0>, 0);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, false, 0>, 0);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, DT, false, 1>, 1);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, false, 1>, 1);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, true, 1>, 1);
  if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_BF16, true, 1>, 1);
  if constexpr (DT != EEP_F32) {
    if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, false, 4>, 4);
    if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, DT, false, 4>, 4);
    if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_F32, true, 4>, 4);
    if (e == hipSuccess) e = allow((const void*)k_grad_tiled<DT, EEP_BF16, true, 4>, 4);
  }
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
      (f.dtype == EEP_BF16 ? allow_grad_lds<EEP_BF16>() : allow_grad_lds<EEP_F32>()) != hipSuccess ||
      hipMalloc((void**)&g->partial, kPartialBytes) != hipSuccess) {
    (void)hipGetLastError();
    delete g;
    return EEP_ERR_HIP;
  }
  *out = g;
  return EEP_OK;
}

int eep_product_grad_destroy(eep_product_grad* grad) {
  if (!grad) return EEP_OK;
  const hipError_t e = hipDeviceSynchronize(), e2 = hipFree(grad->partial);
  delete grad;
  return e == hipSuccess && e2 == hipSuccess ? EEP_OK : EEP_ERR_HIP;
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
    e = bf16 ? launch_grad_x<EEP_BF16>(a, *grad, st) : launch_grad_x<EEP_F32>(a, *grad, st);
  }
  if (e == hipSuccess && grad_w) {
    a.other = (const uint8_t*)x;
    a.out = (uint8_t*)grad_w;
    a.out_stride = grad->grad_stride;
    const bool out16 = f.grad_w_dtype == EEP_BF16;
    e = bf16 ? (out16 ? launch_grad_w<EEP_BF16, EEP_BF16>(a, *grad, st) : launch_grad_w<EEP_BF16, EEP_F32>(a, *grad, st))
             : (out16 ? launch_grad_w<EEP_F32, EEP_BF16>(a, *grad, st) : launch_grad_w<EEP_F32, EEP_F32>(a, *grad, st));
  }
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

}  // extern "C"
