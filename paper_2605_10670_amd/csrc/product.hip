// The experts' product: the rows of every slot times the slot's weights, grouped by the offsets that the layout
// left in device memory.
//
// All kernels work on the transposed product: the matrix cores' rows are rows of the weights (features of y), their
// columns are tokens.  A lane then holds four neighbouring features of ONE token: it needs one scale of x and one of w
// per block, and stores 8 or 16 bytes of a row of y.  Whatever the type, a step is 128 bytes along in_features, of which lane
// l takes 16 bytes of row l % 16 at 16 * (l / 16) and 16 more 64 bytes on, of both operands alike: a product of sums
// does not ask in which order its terms come, so the matrix cores' own order of k plays no part.
#include <math.h>

#include <new>
#include <type_traits>

#include "eep_internal.hpp"
#include "numbers.hpp"
#include "rows.hpp"
#include "tiles.hpp"

struct eep_product {
  eep_product_config cfg;
  int64_t slot_stride, scale_stride;  // bytes
  int cus;                            // of the device
  // where y is codes, else NULL:
  float* values;      // of y before its scales are known, kFewGroups of k_product_few
  uint32_t* arrived;  // how many workgroups of a group have theirs there; zero between calls
};

namespace eep {

constexpr int kStepBytes = 128;  // along in_features
constexpr int kScaleBlock = 128;

struct ProductArgs {
  const uint8_t *x, *w;
  const float *x_scale, *w_scale;
  const int32_t* offset;
  uint8_t* y;
  float* y_scale;
  int rows, slots;
  int row_bytes;  // of x and w
  int features;   // of y
  int feature_tiles;
  int64_t slot_stride, scale_stride;
};

// 32 bytes a lane of a 16-row operand: two chunks of 16.
struct Frag {
  u32x4 c[2];
};

// 16 e4m3 codes as bf16, which holds them exactly.
__device__ __forceinline__ void widen(const u32x4& c, bf16x8 (&out)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, true);
    out[i >> 1][4 * (i & 1)] = lo[0];
    out[i >> 1][4 * (i & 1) + 1] = lo[1];
    out[i >> 1][4 * (i & 1) + 2] = hi[0];
    out[i >> 1][4 * (i & 1) + 3] = hi[1];
  }
}

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

// Codes are multiplied as bf16, of which the matrix cores keep every product: their 8-bit forms line the products of
// 8 neighbouring k up with the largest of them and keep 13 bits below its first (measured with single products
// beside a large one; across the eights nothing is lost), so that 448 * 448 - 448 * 448 + 1 is 0 there.  On normally distributed
// rows a sum of 128 then is 1.3e-5 off (2-norm), and 5.4e-5 with wider ones; as bf16 1e-8 and 7e-8.  What that costs where the matrix
// cores are the bound: 4096 rows 2048 -> 7168 through one matrix 126 us, 67 with the 8-bit forms.
//
// One block of 128: p[m] + w[m] * x.
template <int M>
__device__ __forceinline__ void multiply_codes(const Frag (&w)[M], const Frag& x, f32x4 (&p)[M]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    bf16x8 xv[2];
    widen(x.c[j], xv);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8 wv[2];
      widen(w[m].c[j], wv);
#pragma unroll
      for (int i = 0; i < 2; ++i) p[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], xv[i], p[m], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);  // (what is widened ahead of time takes registers)
  }
}

// The chunks of a row's last bytes; `left` of them from the first chunk on, the rest zeros.
__device__ __forceinline__ Frag load_tail(const uint8_t* from, int left) {
  Frag f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f.c[j] = u32x4{0, 0, 0, 0};
    if (j * 64 < left) f.c[j] = *(const u32x4*)(from + j * 64);
  }
  return f;
}

// load(buffer, step) and multiply(buffer) over the steps [begin, end), AHEAD of them under way.
template <int AHEAD, class Load, class Multiply>
__device__ __forceinline__ void stream(int begin, int end, Load load, Multiply multiply) {
  if (begin >= end) return;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load(u, begin + u < end ? begin + u : end - 1);
  int s = begin;
  for (; s + 2 * AHEAD <= end; s += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      multiply(u);
      load(u, s + u + AHEAD);
    }
  }
  // fewer than twice AHEAD steps are left, up to AHEAD of them loaded
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    if (s + u < end) multiply(u);
    if (s + u + AHEAD < end) load(u, s + u + AHEAD);
  }
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (s + u + AHEAD < end) multiply(u);
}

// An operand, ready to be used several times: e4m3 codes are widened to bf16, once.
template <int DT>
struct Operand {
  Frag f;
  __device__ __forceinline__ void set(const Frag& v) { f = v; }
  __device__ __forceinline__ f32x4 times(const Operand& b, f32x4 acc) const { return mma<DT>(f, b.f, acc); }
};
template <>
struct Operand<EEP_FP8_E4M3> {
  bf16x8 v[2][2];
  __device__ __forceinline__ void set(const Frag& f) {
    widen(f.c[0], v[0]);
    widen(f.c[1], v[1]);
  }
  __device__ __forceinline__ f32x4 times(const Operand& b, f32x4 acc) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[i >> 1][i & 1], b.v[i >> 1][i & 1], acc, 0, 0, 0);
    return acc;
  }
};

// v / (1 + exp(-v)) * u, of an exponential that does not overflow (below -88 the quotient would be 0, however large u is)
__device__ __forceinline__ float silu_times(float v, float u) {
  const float e = expf(-fabsf(v));
  return (v < 0.0f ? v * e : v) / (1.0f + e) * u;
}

// Where the `tile`-th tile of TOKENS rows lies: its slot, its first row and the end of the slot's rows.  false: there are
// fewer.  A lane counts the tiles of a run of slots, a wavefront adds them up; all lanes get the answer.
template <int TOKENS>
__device__ __forceinline__ bool find_tile(const ProductArgs& a, int64_t tile, int* slot, int* first, int* end) {
  if (a.offset == nullptr) {
    *slot = 0;
    *first = (int)(tile * TOKENS);
    *end = a.rows;
    return tile * TOKENS < a.rows;
  }
  const int lane = threadIdx.x & 63;
  const int run = (a.slots + 63) / 64;
  const int p0 = lane * run, p1 = p0 + run < a.slots ? p0 + run : a.slots;
  auto bound = [&](int p) {
    const int o = a.offset[p];
    return o < 0 ? 0 : o > a.rows ? a.rows : o;
  };
  int mine = 0;
  if (p0 < p1) {
    int lo = bound(p0);
    for (int p = p0; p < p1; ++p) {
      const int hi = bound(p + 1);
      if (hi > lo) mine += (hi - lo + TOKENS - 1) / TOKENS;
      lo = hi;
    }
  }
  int upto = mine;  // inclusive sum over the lanes
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  const uint64_t behind = __ballot((int64_t)upto > tile);
  if (behind == 0) return false;
  const int owner = __builtin_ctzll(behind);
  int found[3] = {0, 0, 0};
  if (lane == owner) {
    int64_t left = tile - (upto - mine);
    int lo = bound(p0);
    for (int p = p0; p < p1; ++p) {
      const int hi = bound(p + 1);
      const int n = hi > lo ? (hi - lo + TOKENS - 1) / TOKENS : 0;
      if (left < n) {
        found[0] = p;
        found[1] = lo + (int)left * TOKENS;
        found[2] = hi;
        break;
      }
      left -= n;
      lo = hi;
    }
  }
  *slot = __builtin_amdgcn_readlane(found[0], owner);
  *first = __builtin_amdgcn_readlane(found[1], owner);
  *end = __builtin_amdgcn_readlane(found[2], owner);
  return true;
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
// and each stores 16 bytes, so that a row of y gets 64 at once.  n: the first of the 32 features.
__device__ __forceinline__ void store_tiles(uint8_t* y, int64_t row, int features, int n, int part, bool in_rows,
                                            const f32x4& a, const f32x4& b) {
  const auto low = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[0], a[1]), pack_bf16x2(b[0], b[1]), false, false);
  const auto high = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[2], a[3]), pack_bf16x2(b[2], b[3]), false, false);
  n += (part & 1) * 16 + (part >> 1) * 8;
  if (in_rows && n < features) *(u32x4*)(y + (row * features + n) * 2) = u32x4{low[0], high[0], low[1], high[1]};
}

// ---------------------------------------------------------------------------
// a row or so a slot: the weights go straight to registers.
//
// A workgroup of 8 wavefronts has 16 rows of one slot and 128 features of y with the gate, 256 without: each wavefront two
// matrix-core tiles of 16 weight rows, with the gate the two factors of 16 features.  No weight is used by two
// wavefronts, so nothing of them goes through LDS; the rows of x come from the caches.  Bound by HBM: 16 tokens of 144 slots bf16
// 4096 -> 2 x 1024 252 us (5.7 TB/s), 256 tokens of 288 slots fp8 7168 -> 2 x 2048 1.48 ms (5.7 TB/s); with loads two steps ahead and
// one workgroup to a CU 255 us and 1.52 ms.
// ---------------------------------------------------------------------------
constexpr int kThinTokens = 16, kThinWaves = 8;
template <int DT, int YT, bool GATE>
__global__ __launch_bounds__(64 * kThinWaves, 4) void k_product_thin(ProductArgs a, int64_t first_tile) {
  // steps under way; with the registers that widening takes, as many as leave two workgroups to a CU
  constexpr int kAhead = DT == EEP_FP8_E4M3 ? 3 : 4;
  __shared__ uint32_t s_top[kThinWaves][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, part = lane >> 4;
  const int64_t work = first_tile + blockIdx.x;
  const int64_t row_tile = work / a.feature_tiles;
  const int feature_tile = (int)(work - row_tile * a.feature_tiles);
  int slot, row0, end;
  if (!find_tile<kThinTokens>(a, row_tile, &slot, &row0, &end)) return;

  const int weight_rows = GATE ? 2 * a.features : a.features;
  int n0[2];  // first weight row of the wavefront's two tiles
  if constexpr (GATE) {
    n0[0] = (feature_tile * kThinWaves + wave) * 16;
    n0[1] = n0[0] + a.features;
  } else {
    n0[0] = (feature_tile * kThinWaves + wave) * 32;
    n0[1] = n0[0] + 16;
  }
  // rows past the end are read as the last one; their results are not stored
  const uint8_t* from[3];  // the tiles' first rows, and where the lane reads from there
  uint32_t at[3];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int first = n0[m] < weight_rows ? n0[m] : weight_rows - 1;
    const int n = n0[m] + col < weight_rows ? n0[m] + col : weight_rows - 1;
    from[m] = a.w + slot * a.slot_stride + (int64_t)first * a.row_bytes;
    at[m] = (uint32_t)(n - first) * (uint32_t)a.row_bytes + part * 16;
  }
  const int token = row0 + col < end ? row0 + col : end - 1;
  from[2] = a.x + (int64_t)row0 * a.row_bytes;
  at[2] = (uint32_t)(token - row0) * (uint32_t)a.row_bytes + part * 16;
  const int steps = a.row_bytes / kStepBytes;
  [[maybe_unused]] const int tail = a.row_bytes - steps * kStepBytes;  // bytes, a multiple of 16; 0 for fp8
  const float* sx = nullptr;
  const float* sw[2] = {nullptr, nullptr};
  if constexpr (DT == EEP_FP8_E4M3) {
    sx = a.x_scale + (int64_t)token * steps;
    const float* slot_scale = (const float*)((const uint8_t*)a.w_scale + slot * a.scale_stride);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int n = n0[m] < weight_rows ? n0[m] : weight_rows - 1;
      sw[m] = slot_scale + (int64_t)(n / kScaleBlock) * steps;
    }
  }

  f32x4 acc[2] = {};
  Frag f[kAhead][3];
  float xs[kAhead], ws[kAhead][2];
  auto load = [&](int buffer, int s) {
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int j = 0; j < 2; ++j) f[buffer][m].c[j] = *(const u32x4*)(from[m] + (at[m] + (uint32_t)(s * kStepBytes + j * 64)));
    if constexpr (DT == EEP_FP8_E4M3) {
      xs[buffer] = sx[s];
#pragma unroll
      for (int m = 0; m < 2; ++m) ws[buffer][m] = sw[m][s];
    }
  };
  auto multiply = [&](int buffer) {
    if constexpr (DT == EEP_FP8_E4M3) {
      f32x4 p[2] = {};
      multiply_codes<2>({f[buffer][0], f[buffer][1]}, f[buffer][2], p);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float scale = xs[buffer] * ws[buffer][m];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = fmaf(p[m][i], scale, acc[m][i]);
      }
    } else {
#pragma unroll
      for (int m = 0; m < 2; ++m) acc[m] = mma<DT>(f[buffer][m], f[buffer][2], acc[m]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  stream<kAhead>(0, steps, load, multiply);
  if constexpr (DT != EEP_FP8_E4M3) {
    if (tail != 0) {
      Frag t[3];
#pragma unroll
      for (int m = 0; m < 3; ++m) t[m] = load_tail(from[m] + (at[m] + (uint32_t)(steps * kStepBytes)), tail - part * 16);
#pragma unroll
      for (int m = 0; m < 2; ++m) acc[m] = mma<DT>(t[m], t[2], acc[m]);
    }
  }

  const bool in_rows = row0 + col < end;
  const int64_t out_row = (int64_t)(row0 + col) * a.features;
  if constexpr (GATE) {
    const int n = n0[0] + part * 4;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = silu_times(acc[0][i], acc[1][i]);
    if constexpr (YT == EEP_FP8_E4M3) {
      uint32_t top = top_magnitude<4>(v);
      top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
      if (part == 0) s_top[wave][col] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kThinWaves; ++w) top = max(top, s_top[w][col]);
      const float scale = scale_of(top);
      if (in_rows) {
        *(uint32_t*)(a.y + out_row + n) = codes4(v[0], v[1], v[2], v[3], scale);
        if (wave == 0 && part == 0) a.y_scale[(int64_t)(row0 + col) * a.feature_tiles + feature_tile] = scale;
      }
    } else {
      if (in_rows && n < a.features) store4<YT>(a.y, out_row + n, v);
    }
  } else {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int n = n0[m] + part * 4;
      const float v[4] = {acc[m][0], acc[m][1], acc[m][2], acc[m][3]};
      if (in_rows && n < a.features) store4<YT>(a.y, out_row + n, v);
    }
  }
}

// ---------------------------------------------------------------------------
// so few rows that the others would leave CUs idle: 16 * M weight rows by 16 * TN tokens a workgroup.
//
// The workgroup's 8 wavefronts divide in_features and add their sums up in LDS, in the order of the parts; with the gate a
// tile's 16 rows are 8 of either factor.  Codes need the largest of 128 features, which are 16 tiles' here: each leaves
// its values in memory, past the L2s, which do not see one another's writes, and the last to arrive makes the codes of
// all.  (Its loads look past the caches one by one; a fence would empty them for everybody.)  Bound by latency: one token through
// 7168 -> 2 x 2048 fp8 to codes 12.2 us, of which the rows' trip and the sums are 7, the values' and the codes' 5; 2048 -> 7168
// to bf16 6.7.  (In_features divided between workgroups instead, the last to arrive adding up: 15.0 and 9.9.)
// ---------------------------------------------------------------------------
constexpr int kFewGroups = 256;  // groups of 16 tokens by 128 features that the workspace holds

// Two workgroups to a CU, or one with twice the registers.
constexpr bool few_alone(int m, int tn) { return m * tn > 2; }

template <int DT, int YT, bool GATE, int M, int TN>
__global__ __launch_bounds__(64 * kThinWaves, few_alone(M, TN) ? 2 : 4) void k_product_few(ProductArgs a, float* values, uint32_t* arrived) {
  constexpr bool kCodes = DT == EEP_FP8_E4M3;
  constexpr int kAhead = few_alone(M, TN) ? (M + TN > 8 ? 1 : 16 / (M + TN)) : M + TN == 2 ? 4 : 3;  // steps under way, as many as there are registers for
  constexpr int kFeatures = GATE ? 8 : 16;
  __shared__ f32x4 s_sum[kThinWaves][M * TN][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, part = lane >> 4;
  const int row_tile = blockIdx.x / a.feature_tiles, feature_tile = blockIdx.x - row_tile * a.feature_tiles;
  int slot, row0, end;
  if (!find_tile<kThinTokens * TN>(a, row_tile, &slot, &row0, &end)) return;

  const int row_steps = a.row_bytes / kStepBytes;
  const int begin = row_steps * wave / kThinWaves, steps = row_steps * (wave + 1) / kThinWaves;
  const uint8_t* w_base = a.w + slot * a.slot_stride;
  const uint8_t* x_base = a.x + (int64_t)row0 * a.row_bytes;
  const float *w_scale = nullptr, *x_scale = nullptr;
  uint32_t w_at[M], x_at[TN], w_scale_at[M], x_scale_at[TN];
  if constexpr (kCodes) {
    w_scale = (const float*)((const uint8_t*)a.w_scale + slot * a.scale_stride);
    x_scale = a.x_scale + (int64_t)row0 * row_steps;
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int n0 = (feature_tile * M + m) * kFeatures;
    const int second = GATE && col >= kFeatures ? 1 : 0;  // of the factors
    int n = n0 + col - second * kFeatures;
    n = n < a.features ? n : a.features - 1;
    w_at[m] = (uint32_t)(n + second * a.features) * (uint32_t)a.row_bytes + part * 16;
    // the scale is that of the lane's sums: with the gate those of parts 2 and 3 belong to the other factor
    const int row = (n0 < a.features ? n0 : 0) + (GATE && part >= 2 ? a.features : 0);
    w_scale_at[m] = (uint32_t)(row / kScaleBlock * row_steps);
  }
#pragma unroll
  for (int t = 0; t < TN; ++t) {
    const int token = row0 + t * 16 + col < end ? t * 16 + col : end - 1 - row0;
    x_at[t] = (uint32_t)token * (uint32_t)a.row_bytes + part * 16;
    x_scale_at[t] = (uint32_t)(token * row_steps);
  }

  f32x4 acc[M][TN] = {};
  Frag w[kAhead][M], x[kAhead][TN];
  float xs[kAhead][TN], ws[kAhead][M];
  auto load = [&](int buffer, int s) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t at = (uint32_t)(s * kStepBytes + j * 64);
#pragma unroll
      for (int m = 0; m < M; ++m) w[buffer][m].c[j] = *(const u32x4*)(w_base + (w_at[m] + at));
#pragma unroll
      for (int t = 0; t < TN; ++t) x[buffer][t].c[j] = *(const u32x4*)(x_base + (x_at[t] + at));
    }
    if constexpr (kCodes) {
#pragma unroll
      for (int m = 0; m < M; ++m) ws[buffer][m] = w_scale[w_scale_at[m] + (uint32_t)s];
#pragma unroll
      for (int t = 0; t < TN; ++t) xs[buffer][t] = x_scale[x_scale_at[t] + (uint32_t)s];
    }
  };
  auto multiply = [&](int buffer) {
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      if constexpr (kCodes) {
        f32x4 p[M] = {};
        multiply_codes<M>(w[buffer], x[buffer][t], p);
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const float scale = xs[buffer][t] * ws[buffer][m];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][t][i] = fmaf(p[m][i], scale, acc[m][t][i]);
        }
      } else {
#pragma unroll
        for (int m = 0; m < M; ++m) acc[m][t] = mma<DT>(w[buffer][m], x[buffer][t], acc[m][t]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  stream<kAhead>(begin, steps, load, multiply);
  if constexpr (!kCodes) {
    const int tail = a.row_bytes - row_steps * kStepBytes;
    if (tail != 0 && wave == kThinWaves - 1) {
      const uint32_t at = (uint32_t)(row_steps * kStepBytes);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const Frag wt = load_tail(w_base + (w_at[m] + at), tail - part * 16);
#pragma unroll
        for (int t = 0; t < TN; ++t) acc[m][t] = mma<DT>(wt, load_tail(x_base + (x_at[t] + at), tail - part * 16), acc[m][t]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int t = 0; t < TN; ++t) s_sum[wave][m * TN + t][lane] = acc[m][t];
  __syncthreads();
  // a wavefront finishes a tile
  if (wave >= M * TN) return;
  const int m = wave / TN, t = wave % TN;
  const int n0 = (feature_tile * M + m) * kFeatures;
  if (n0 >= a.features) return;
  f32x4 sum = s_sum[0][wave][lane];
#pragma unroll
  for (int other = 1; other < kThinWaves; ++other) sum += s_sum[other][wave][lane];

  const int64_t row = row0 + t * 16 + col;
  const bool in_rows = row < end;
  float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  if constexpr (GATE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = silu_times(v[i], __shfl_xor(v[i], 32, 64));
  }
  const bool has = in_rows && (!GATE || part < 2);  // (with the gate the other parts have nothing of their own now)
  const int n = n0 + part * 4;
  if constexpr (YT != EEP_FP8_E4M3) {
    if (has && n < a.features) store4<YT>(a.y, row * a.features + n, v);
  } else {
    constexpr int kMembers = kScaleBlock / kFeatures;  // (whole groups: features are a multiple of 128)
    const int blocks = a.features / kScaleBlock, block = n0 / kScaleBlock;
    const int group = (row_tile * TN + t) * blocks + block;
    float* all = values + ((int64_t)group * kThinTokens + col) * kScaleBlock;
    if (has) store_row((u32x4*)(all + n % kScaleBlock), __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they are where all workgroups see them
    uint32_t before = 0;
    if (lane == 0) before = __hip_atomic_fetch_add(&arrived[group], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane(before) != kMembers - 1) return;
    if (lane == 0) __hip_atomic_store(&arrived[group], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!in_rows) return;  // (lanes of one token go together)
    // a lane has every fourth 8 features of a token
    float q[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t d = __hip_atomic_load((const uint64_t*)(all + (i * 4 + part) * 8) + j, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT);
        q[i][2 * j] = __uint_as_float((uint32_t)d);
        q[i][2 * j + 1] = __uint_as_float((uint32_t)(d >> 32));
      }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, top_magnitude<8>(q[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    const float scale = scale_of(top);
    if (part == 0) a.y_scale[row * blocks + block] = scale;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(u32x2*)(a.y + row * a.features + block * kScaleBlock + (i * 4 + part) * 8) =
          u32x2{codes4(q[i][0], q[i][1], q[i][2], q[i][3], scale), codes4(q[i][4], q[i][5], q[i][6], q[i][7], scale)};
  }
}

// ---------------------------------------------------------------------------
// many rows a slot: tiles through LDS.
//
// A workgroup of 8 wavefronts has 256 weight rows (with the gate 128 of each factor) by 64 * TT tokens; of these a wavefront
// holds the sums of 128 by 64, 64 by 64 or 64 by 32, near a square, so that it reads few rows of a step for them.  A step's rows go from memory to LDS without passing through registers, STAGES - 1 steps ahead; a row's eight
// 16-byte chunks lie in LDS at their number XOR the row's, so that the 16 rows of a tile are read without bank
// conflicts although each begins at the same bank.
//
// The workgroups stay: each goes through its share of the work items, an item being a tile.  Workgroups of one XCD
// (every eighth) have neighbouring items, those of one slot with the row tiles innermost: what runs at a time
// shares weights and rows in that XCD's L2.
//
// Measured: 4096 tokens of 288 slots fp8 2048 -> 7168 to bf16 1238 us (3.9 TB/s, 0.78 PFLOP/s), 4096 rows
// through one such matrix 126 us (0.95 PFLOP/s), bf16 1408 -> 2880 to fp32, 35856 rows in 120 slots, 415 us (0.70 PFLOP/s, 3.5 TB/s),
// 16384 tokens fp8 7168 -> 2 x 2048 to codes 7.8 to 8.3 ms (0.95 PFLOP/s).  Codes are bound by instructions: a SIMD's matrix and vector
// instructions take their times one after the other (two wavefronts of products with two vector instructions each ran
// in the sum of both, not the larger), and a step of a wavefront has 64 products, 128 instructions that widen codes and
// 64 that scale the sums.
// ---------------------------------------------------------------------------
constexpr int kTiledWaves = 8, kTiledRows = 256;
constexpr int kTiledThreads = 64 * kTiledWaves;
__host__ __device__ constexpr int tiled_across(int tt) { return tt == 4 ? 2 : 4; }  // wavefronts side by side on the weight rows
__host__ __device__ constexpr int tiled_stages(int tt) { return tt == 4 ? 2 : 3; }
// Codes' scales come four steps at a time: a token's side by side, behind them those of two blocks of weight rows.
constexpr int kScaleSteps = 4, kScaleBuffers = 3;
constexpr int kWeightStage = kTiledRows * kStepBytes;
__host__ __device__ constexpr int tiled_scale_bytes(int tt) { return 64 * tt * kScaleSteps * 4 + 256; }
__host__ __device__ constexpr int tiled_lds_bytes(bool codes, int tt) {
  return tiled_stages(tt) * (kWeightStage + 64 * tt * kStepBytes) +
         (codes ? kScaleBuffers * tiled_scale_bytes(tt) : 0) + tiled_across(tt) * 64 * tt * 4;
}

typedef const __attribute__((address_space(1))) void global_void;

template <int DT, int YT, bool GATE, int TT>
__global__ __launch_bounds__(kTiledThreads, 2) void k_product_tiled(ProductArgs a) {
  constexpr int kWM = tiled_across(TT), kWN = kTiledWaves / kWM;
  constexpr int kA = kTiledRows / 16 / kWM, kB = 4 * TT / kWN;  // tiles of 16 weight rows and of 16 tokens a wavefront
  constexpr int kStages = tiled_stages(TT), kTokens = 64 * TT;
  constexpr bool kCodes = DT == EEP_FP8_E4M3;
  constexpr int kXStage = kTokens * kStepBytes, kScaleBytes = tiled_scale_bytes(TT);
  constexpr int kWeightLoads = kTiledRows / 8 / kTiledWaves, kXLoads = kTokens / 8 / kTiledWaves;  // of 8 rows each, a wavefront and step
  constexpr bool kEarly = TT == 4;  // the tokens' rows are fetched as soon as all wavefronts have read theirs
  constexpr int kScaleLoads = 4 * TT >= kTiledWaves ? 4 * TT / kTiledWaves : 1;  // of 16 tokens each, a wavefront
  extern __shared__ __align__(1024) uint8_t lds[];
  uint8_t* const x_lds = lds + kStages * kWeightStage;
  uint8_t* const scale_lds = x_lds + kStages * kXStage;
  uint32_t* s_top = (uint32_t*)(scale_lds + (kCodes ? kScaleBuffers * kScaleBytes : 0));  // [kWM][kTokens]

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % kWM, wn = wave / kWM;
  const int col = lane & 15, part = lane >> 4;

  TileMap<kTokens> map;
  map.make(a);
  const int64_t items = (int64_t)map.total * a.feature_tiles;
  // the items of this workgroup: those of its XCD, every so manieth
  const int xcds = gridDim.x % 8 == 0 ? 8 : 1;
  const int xcd = blockIdx.x % xcds, seat = blockIdx.x / xcds, seats = gridDim.x / xcds;
  const int64_t from = items * xcd / xcds, to = items * (xcd + 1) / xcds;

  const int weight_rows = GATE ? 2 * a.features : a.features;
  const int full_steps = a.row_bytes / kStepBytes;
  const int tail = a.row_bytes - full_steps * kStepBytes;
  const int steps = full_steps + (tail != 0 ? 1 : 0);

  // what the lane loads: 16 bytes of row `lane / 8` of eight
  const int load_row = lane >> 3, load_chunk = (lane & 7) ^ load_row;
  const int tail_chunk = load_chunk * 16 < tail ? load_chunk : 0;  // past the row's end: anything of it
  // what it reads of a tile of 16 rows: two chunks
  const int read_at = col * kStepBytes + ((part ^ (col & 7)) << 4);

  struct Tile {
    int slot, feature_tile, first, end;
  };
  Tile t = {}, next = {};
  const uint8_t *w_base, *x_base;                   // of the tiles whose rows are loaded
  uint32_t w_row_at[kWeightLoads], x_row_at[kXLoads];  // first byte of the lane's rows from there
  const float *x_scale = nullptr, *w_scale = nullptr;
  uint32_t scale_at[kScaleLoads];                   // and of its tokens' scales
  auto aim_weights = [&](const Tile& tile) {
    const int half = GATE ? 128 : 256;  // weight rows in one piece
    const int n0 = tile.feature_tile * half;
    const int piece = GATE && wave >= kTiledWaves / 2 ? 1 : 0;
    w_base = a.w + tile.slot * a.slot_stride + (int64_t)(n0 + piece * a.features) * a.row_bytes;
#pragma unroll
    for (int i = 0; i < kWeightLoads; ++i) {
      const int r = (wave * kWeightLoads + i) * 8 + load_row - piece * half;
      w_row_at[i] = (uint32_t)(n0 + r < a.features ? r : a.features - 1 - n0) * (uint32_t)a.row_bytes;
    }
    if constexpr (kCodes) {
      x_scale = a.x_scale + (int64_t)tile.first * steps;
#pragma unroll
      for (int i = 0; i < kScaleLoads; ++i) {
        int r = (wave * kScaleLoads + i) % (4 * TT) * 16 + (lane >> 2);
        r = tile.first + r < tile.end ? r : tile.end - 1 - tile.first;
        scale_at[i] = (uint32_t)(r > 0 ? r : 0) * (uint32_t)steps;
      }
      // blocks of 128 weight rows: one of each factor with the gate, else the two of the tile, if it has two
      const int block = GATE ? tile.feature_tile : 2 * tile.feature_tile;
      w_scale = (const float*)((const uint8_t*)a.w_scale + tile.slot * a.scale_stride) + (int64_t)block * steps;
    }
  };
  auto aim_tokens = [&](const Tile& tile) {
    x_base = a.x + (int64_t)tile.first * a.row_bytes;
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
      int r = (wave * kXLoads + i) * 8 + load_row;
      r = tile.first + r < tile.end ? r : tile.end - 1 - tile.first;
      x_row_at[i] = (uint32_t)(r > 0 ? r : 0) * (uint32_t)a.row_bytes;
    }
  };
  const int last_block = (weight_rows - 1) / kScaleBlock;
  auto fetch_scales = [&](const Tile& tile, int chunk, uint8_t* to_lds) {
    int q = chunk * kScaleSteps + (lane & 3);
    q = q < steps ? q : steps - 1;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
      __builtin_amdgcn_global_load_lds((global_void*)(x_scale + (scale_at[i] + (uint32_t)q)),
                                       (lds_void*)(to_lds + (wave * kScaleLoads + i) % (4 * TT) * 256), 4, 0, 0);
    const int second = GATE ? a.features / kScaleBlock : 2 * tile.feature_tile < last_block ? 1 : 0;
    __builtin_amdgcn_global_load_lds((global_void*)(w_scale + (uint32_t)((lane & 4 ? second * steps : 0) + q)),
                                     (lds_void*)(to_lds + kTokens * 16), 4, 0, 0);
  };
  auto bytes_in = [&](int step) {
    return (uint32_t)(step * kStepBytes + (step < full_steps ? load_chunk : tail_chunk) * 16);
  };
  auto fetch_weights = [&](int step, uint8_t* to_lds) {
    const uint32_t at = bytes_in(step);
#pragma unroll
    for (int i = 0; i < kWeightLoads; ++i)
      __builtin_amdgcn_global_load_lds((global_void*)(w_base + (w_row_at[i] + at)),
                                       (lds_void*)(to_lds + (wave * kWeightLoads + i) * 8 * kStepBytes), 16, 0, 0);
  };
  auto fetch_tokens = [&](int step, uint8_t* to_lds) {
    const uint32_t at = bytes_in(step);
#pragma unroll
    for (int i = 0; i < kXLoads; ++i)
      __builtin_amdgcn_global_load_lds((global_void*)(x_base + (x_row_at[i] + at)),
                                       (lds_void*)(to_lds + (wave * kXLoads + i) * 8 * kStepBytes), 16, 0, 0);
  };

  int64_t item = from + seat;
  if (item >= to) return;
  map.find(a, item, &t.slot, &t.feature_tile, &t.first, &t.end);
  aim_weights(t);
  aim_tokens(t);
  // The steps of all tiles are one stream, fetched ahead (no row is shorter than that).  Behind its end the last step
  // is fetched again, to no purpose, so that the number of loads under way is always the same.
  int64_t fetch_item = item;
  int w_step = 0, x_step = 0;  // to be fetched next
  bool more = true;
  uint8_t* chunk = scale_lds;  // where the scales of the step are
  auto behind = [&](uint8_t* p, int n) {
    p += n * kScaleBytes;
    return p < scale_lds + kScaleBuffers * kScaleBytes ? p : p - kScaleBuffers * kScaleBytes;
  };
  // At the top of step s: the scales of the next four steps, and the next tile, once the fetches have come to them.
  auto look_ahead = [&](int s) {
    if constexpr (kCodes) {
      if ((s & 3) == 0 && s + kScaleSteps < steps) fetch_scales(t, s / kScaleSteps + 1, behind(chunk, 1));
    }
    if (w_step == steps) {
      more = fetch_item + seats < to;
      if (more) {
        fetch_item += seats;
        map.find(a, fetch_item, &next.slot, &next.feature_tile, &next.first, &next.end);
        aim_weights(next);
        if constexpr (kCodes) fetch_scales(next, 0, behind(chunk, (steps - 1) / kScaleSteps - s / kScaleSteps + 1));
      }
      w_step = more ? 0 : steps - 1;
    }
    if (x_step == steps) {
      if (more) aim_tokens(next);
      x_step = more ? 0 : steps - 1;
    }
  };
  if constexpr (kCodes) fetch_scales(t, 0, chunk);
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    fetch_tokens(x_step++, x_lds + s * kXStage);
    fetch_weights(w_step++, lds + s * kWeightStage);
  }

  // What a step begins with: the tokens' rows, the first weight rows, the scales; read while the step before ends.
  Frag b_raw[kB], a_raw;
  [[maybe_unused]] float token_scale[kB], row_scale[2];
  uint8_t *stage = lds, *x_stage = x_lds;  // of the step
  auto read = [&](const uint8_t* from_lds, int tile_row) {
    Frag f;
    f.c[0] = *(const u32x4*)(from_lds + tile_row * kStepBytes + read_at);
    f.c[1] = *(const u32x4*)(from_lds + tile_row * kStepBytes + (read_at ^ 64));
    return f;
  };
  auto row_of_tile = [&](int f) {
    return GATE ? f / (kA / 2) * 128 + wm * (128 / kWM) + f % (kA / 2) * 16 : wm * (256 / kWM) + f * 16;
  };
  auto read_scales = [&](int s) {
    if constexpr (kCodes) {
      const float* scales = (const float*)chunk + (s & 3);
#pragma unroll
      for (int j = 0; j < kB; ++j) token_scale[j] = scales[((wn * kB + j) * 16 + col) * 4];
      row_scale[0] = scales[kTokens * 4 + (GATE ? 0 : wm / (kWM / 2) * 4)];
      if constexpr (GATE) row_scale[1] = scales[kTokens * 4 + 4];
    }
  };
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * (kWeightLoads + kXLoads)) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_scales(0);
#pragma unroll
  for (int j = 0; j < kB; ++j) b_raw[j] = read(x_stage, (wn * kB + j) * 16);
  a_raw = read(stage, row_of_tile(0));

  for (;;) {
    f32x4 acc[kA][kB];
#pragma unroll
    for (int f = 0; f < kA; ++f)
#pragma unroll
      for (int j = 0; j < kB; ++j) acc[f][j] = f32x4{0, 0, 0, 0};

    auto step = [&](int s, auto is_cut) {
      constexpr bool kCut = decltype(is_cut)::value;  // the last step of rows that end within it
      auto ready = [&](Frag f) {
        if constexpr (kCut) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
            if (j * 64 + part * 16 >= tail) f.c[j] = u32x4{0, 0, 0, 0};
        }
        Operand<DT> o;
        o.set(f);
        return o;
      };
      Operand<DT> b[kB];
#pragma unroll
      for (int j = 0; j < kB; ++j) b[j] = ready(b_raw[j]);
      [[maybe_unused]] float scale[GATE ? 2 : 1][kB];
      if constexpr (kCodes) {
#pragma unroll
        for (int j = 0; j < kB; ++j) {
          scale[0][j] = token_scale[j] * row_scale[0];
          if constexpr (GATE) scale[1][j] = token_scale[j] * row_scale[1];
        }
      }
      // codes: the block's sums of a tile are multiplied by the scales and added while the next ones are multiplied
      constexpr int kBehind = 2;
      [[maybe_unused]] f32x4 block[kBehind + 1];
      // the i-th tile: weight rows by weight rows, then the last two of them side by side
      constexpr int kPairs = (kA - 2) * kB;
      auto tile_f = [](int i) { return i < kPairs ? i / kB : kA - 2 + (i & 1); };
      auto tile_j = [](int i) { return i < kPairs ? i % kB : (i - kPairs) / 2; };
      auto add_block = [&](int i) {
        if constexpr (kCodes) {
          const int f = tile_f(i), j = tile_j(i);
#pragma unroll
          for (int n = 0; n < 4; ++n)
            acc[f][j][n] = fmaf(block[i % (kBehind + 1)][n], scale[GATE ? f / (kA / 2) : 0][j], acc[f][j][n]);
        }
      };
      auto multiply = [&](int i, const Operand<DT>& av) {
        const int f = tile_f(i), j = tile_j(i);
        if constexpr (kCodes) {
          block[i % (kBehind + 1)] = av.times(b[j], f32x4{0, 0, 0, 0});
          if (i >= kBehind) add_block(i - kBehind);
          __builtin_amdgcn_sched_barrier(0);
        } else {
          acc[f][j] = av.times(b[j], acc[f][j]);
        }
      };
      Operand<DT> last[2];
#pragma unroll
      for (int f = 0; f < kA - 2; ++f) {
        const Operand<DT> av = ready(a_raw);
        a_raw = read(stage, row_of_tile(f + 1));
#pragma unroll
        for (int j = 0; j < kB; ++j) multiply(f * kB + j, av);
        if constexpr (!kCodes) __builtin_amdgcn_sched_barrier(0);
        if (kEarly && f == 2) {
          // All wavefronts have their tokens' rows in registers (only the two reads of the next weight rows may be under
          // way): the stage of these is filled again.
          asm volatile("s_waitcnt lgkmcnt(2)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          fetch_tokens(x_step++, x_stage);
        }
      }
      last[0] = ready(a_raw);
      last[1] = ready(read(stage, row_of_tile(kA - 1)));
      // This wavefront has read all it needs of the stage.  Once all have, and the next step's rows are there (no more than
      // the fetches behind them are under way), the stage may be filled again and the next step's first operands are read.
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kEarly ? kXLoads : (kStages - 2) * (kWeightLoads + kXLoads)) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (!kEarly) fetch_tokens(x_step++, x_stage);
      fetch_weights(w_step++, stage);
      uint8_t* following = stage + kWeightStage < lds + kStages * kWeightStage ? stage + kWeightStage : lds;
      uint8_t* x_following = x_stage + kXStage < x_lds + kStages * kXStage ? x_stage + kXStage : x_lds;
      a_raw = read(following, row_of_tile(0));
#pragma unroll
      for (int j = 0; j < kB; ++j) {
        multiply(kPairs + 2 * j, last[0]);
        multiply(kPairs + 2 * j + 1, last[1]);
        b_raw[j] = read(x_following, (wn * kB + j) * 16);
        if constexpr (!kCodes) __builtin_amdgcn_sched_barrier(0);
      }
      const int upcoming = s + 1 < steps ? s + 1 : 0;
      if ((upcoming & 3) == 0) chunk = behind(chunk, 1);
      read_scales(upcoming);
      if constexpr (kCodes) {
#pragma unroll
        for (int i = kA * kB - kBehind; i < kA * kB; ++i) add_block(i);
      }
      stage = following;
      x_stage = x_following;
    };
    for (int s = 0; s < full_steps; ++s) {
      look_ahead(s);
      step(s, std::false_type());
    }
    if constexpr (!kCodes) {
      if (tail != 0) {
        look_ahead(full_steps);
        step(full_steps, std::true_type());
      }
    }

    if constexpr (GATE) {
      const int n0 = t.feature_tile * 128 + wm * (128 / kWM) + part * 4;
      uint32_t top[kB];
#pragma unroll
      for (int j = 0; j < kB; ++j) {
        top[j] = 0;
#pragma unroll
        for (int f = 0; f < kA / 2; ++f) {
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[f][j][i] = v[i] = silu_times(acc[f][j][i], acc[f + kA / 2][j][i]);
          const uint32_t m = top_magnitude<4>(v);
          top[j] = m > top[j] ? m : top[j];
        }
      }
      if constexpr (YT == EEP_FP8_E4M3) {
#pragma unroll
        for (int j = 0; j < kB; ++j) {
          top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 16, 64));
          top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 32, 64));
          if (part == 0) s_top[wm * kTokens + (wn * kB + j) * 16 + col] = top[j];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < kB; ++j) {
          const int at = (wn * kB + j) * 16 + col;
#pragma unroll
          for (int w = 0; w < kWM; ++w) top[j] = max(top[j], s_top[w * kTokens + at]);
          const float scale = scale_of(top[j]);
          const int64_t row = t.first + at;
          if (row < t.end) {
#pragma unroll
            for (int f = 0; f < kA / 2; ++f)
              *(uint32_t*)(a.y + row * a.features + n0 + f * 16) =
                  codes4(acc[f][j][0], acc[f][j][1], acc[f][j][2], acc[f][j][3], scale);
            if (wm == 0 && part == 0) a.y_scale[row * a.feature_tiles + t.feature_tile] = scale;
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < kB; ++j) {
          const int64_t row = t.first + (wn * kB + j) * 16 + col;
          if constexpr (YT == EEP_BF16) {
#pragma unroll
            for (int f = 0; f < kA / 2; f += 2)
              store_tiles(a.y, row, a.features, n0 - part * 4 + f * 16, part, row < t.end, acc[f][j], acc[f + 1][j]);
          } else {
#pragma unroll
            for (int f = 0; f < kA / 2; ++f) {
              const float v[4] = {acc[f][j][0], acc[f][j][1], acc[f][j][2], acc[f][j][3]};
              if (row < t.end && n0 + f * 16 < a.features) store4<YT>(a.y, row * a.features + n0 + f * 16, v);
            }
          }
        }
      }
    } else {
      const int n0 = t.feature_tile * 256 + wm * (256 / kWM) + part * 4;
#pragma unroll
      for (int j = 0; j < kB; ++j) {
        const int64_t row = t.first + (wn * kB + j) * 16 + col;
        if constexpr (YT == EEP_BF16) {
#pragma unroll
          for (int f = 0; f < kA; f += 2)
            store_tiles(a.y, row, a.features, n0 - part * 4 + f * 16, part, row < t.end, acc[f][j], acc[f + 1][j]);
        } else {
#pragma unroll
          for (int f = 0; f < kA; ++f) {
            const float v[4] = {acc[f][j][0], acc[f][j][1], acc[f][j][2], acc[f][j][3]};
            if (row < t.end && n0 + f * 16 < a.features) store4<YT>(a.y, row * a.features + n0 + f * 16, v);
          }
        }
      }
    }
    item += seats;
    if (item >= to) break;
    t = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may still write to LDS when the workgroup is gone
}

// Tiles of `tokens` rows that the slots may have at most.
int64_t most_tiles(int rows, int slots, int tokens) {
  const int64_t touched = rows < slots ? rows : slots;
  return (rows + touched * (tokens - 1)) / tokens;
}

template <int DT, int YT, bool GATE>
hipError_t launch_thin(ProductArgs a, hipStream_t st) {
  constexpr int kThreads = 64 * kThinWaves, kFeatures = GATE ? 16 * kThinWaves : 32 * kThinWaves;
  a.feature_tiles = (a.features + kFeatures - 1) / kFeatures;
  const int64_t work = most_tiles(a.rows, a.slots, kThinTokens) * a.feature_tiles;
  return in_launches(work, max_blocks(kThreads), [&](int64_t first, int64_t n) {
    hipLaunchKernelGGL((k_product_thin<DT, YT, GATE>), dim3((unsigned)n), dim3(kThreads), 0, st, a, first);
    return hipGetLastError();
  });
}

// false: that would be more workgroups than the CUs take at a time, or more groups than the workspace holds, or weights of a
// slot that 32 bits do not span
template <int DT, int YT, bool GATE, int M, int TN>
bool launch_few(const eep_product& p, ProductArgs a, hipStream_t st, hipError_t* e) {
  constexpr int kFeatures = (GATE ? 8 : 16) * M;
  a.feature_tiles = (a.features + kFeatures - 1) / kFeatures;
  const int64_t row_tiles = most_tiles(a.rows, a.slots, kThinTokens * TN), work = row_tiles * a.feature_tiles;
  if (work > (few_alone(M, TN) ? 1 : 2) * p.cus || (int64_t)a.features * (GATE ? 2 : 1) * a.row_bytes >= (int64_t)1 << 32)
    return false;
  if (YT == EEP_FP8_E4M3 && row_tiles * TN * (a.features / kScaleBlock) > kFewGroups) return false;
  hipLaunchKernelGGL((k_product_few<DT, YT, GATE, M, TN>), dim3((unsigned)work), dim3(64 * kThinWaves), 0, st, a, p.values,
                     p.arrived);
  *e = hipGetLastError();
  return true;
}

template <int DT, int YT, bool GATE, int TT>
hipError_t launch_tiled(ProductArgs a, int cus, hipStream_t st) {
  const int features = GATE ? kTiledRows / 2 : kTiledRows;
  a.feature_tiles = (a.features + features - 1) / features;
  const int64_t work = most_tiles(a.rows, a.slots, 64 * TT) * a.feature_tiles;
  hipLaunchKernelGGL((k_product_tiled<DT, YT, GATE, TT>), dim3((unsigned)(work < cus ? work : cus)), dim3(kTiledThreads),
                     tiled_lds_bytes(DT == EEP_FP8_E4M3, TT), st, a);
  return hipGetLastError();
}

// What the tiles of 64 * tt tokens cost, in time: what a step of one takes (us), as often as a CU has one.  A slot's last
// tile is half empty on average.  The same steps are taken for every type; with a tile of one matrix on each CU and 128 steps they measured
// 0.68 / 1.1 / 1.8 in bf16, 1.2 / 1.9 with codes, 2.0 / 3.8 / 7.3 in fp32.
float tiled_cost(int tt, int rows, int slots, int64_t feature_tiles, int cus) {
  const float step = tt == 1 ? 0.95f : tt == 2 ? 1.35f : 2.2f;
  const int touched = rows < slots ? rows : slots;
  float tiles = (float)rows / touched / (64 * tt) + 0.5f;
  if (touched == 1) tiles = (float)((rows + 64 * tt - 1) / (64 * tt));
  const float rounds = (tiles < 1.0f ? 1.0f : tiles) * touched * feature_tiles / cus;
  return step * (rounds < 4.0f ? ceilf(rounds) : rounds);
}

// Rows a slot up to which the thin kernel is chosen: about one; more where the tiles' kernel has codes to widen, which there takes
// the time of the products themselves.  Thin / tiles of 64 tokens, us: 144 slots bf16 4096 -> 2 x 1024, 64 tokens (3.6 rows
// a slot) 464 / 410, 200 tokens (11) 477 / 417; 288 slots 7168 -> 2 x 2048 fp8 to codes, 64 tokens (1.8) 1180 / 1289, 256 (7.1)
// 1482 / 1545, 330 (9.2, where some slots have more than 16 and are read twice) 1557 / 1525, 512 (14.2) 1986 / 1539; 2048 -> 7168 to bf16, 128 tokens
// (3.6) 684 / 760, 256 773 / 790, 330 826 / 797; to fp32, 32 tokens (0.9) 405 / 510.
// fp32 products take the matrix cores 16 times as long as bf16 ones, and tiles of 64 tokens are mostly empty there: 144 slots
// 2048 -> 1024, 200 tokens (11 rows a slot) 291 / 389, 9 slots 4992 -> 4096, 76 rows 209 / 314.
constexpr int thin_mean(int dt) { return dt == EEP_F32 ? 16 : dt == EEP_FP8_E4M3 ? 8 : 1; }

// Are there tiles of 256 tokens?  (widened codes take twice the registers)
constexpr bool tiled_large(int dt) { return dt != EEP_FP8_E4M3; }

// More LDS than a kernel may have by default, for the tiles that a product may be launched with.  On the current device: a kernel has a
// limit on each.
template <int DT, int YT, bool GATE>
hipError_t allow_lds() {
  const auto allow = [](const void* kernel, int tt) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, tiled_lds_bytes(DT == EEP_FP8_E4M3, tt));
  };
  hipError_t e = allow((const void*)k_product_tiled<DT, YT, GATE, 1>, 1);
  if (e == hipSuccess) e = allow((const void*)k_product_tiled<DT, YT, GATE, 2>, 2);
  if constexpr (tiled_large(DT))
    if (e == hipSuccess) e = allow((const void*)k_product_tiled<DT, YT, GATE, 4>, 4);
  return e;
}

template <int DT, int YT, bool GATE>
hipError_t launch_product(const eep_product& p, const ProductArgs& a, hipStream_t st) {
  const int mean = (a.rows + a.slots - 1) / a.slots;  // rows a slot
  hipError_t e = hipSuccess;
  if (mean <= 16) {
    if (launch_few<DT, YT, GATE, 1, 1>(p, a, st, &e) || launch_few<DT, YT, GATE, 2, 1>(p, a, st, &e) ||
        launch_few<DT, YT, GATE, 8, 1>(p, a, st, &e))
      return e;
  } else if (mean <= 32) {
    if (launch_few<DT, YT, GATE, 1, 2>(p, a, st, &e) || launch_few<DT, YT, GATE, 4, 2>(p, a, st, &e)) return e;
  } else if (mean <= 64) {
    if (launch_few<DT, YT, GATE, 1, 4>(p, a, st, &e) || launch_few<DT, YT, GATE, 2, 4>(p, a, st, &e)) return e;
  }
  // (the tiles' stream is as long as three steps at least)
  if (mean <= thin_mean(DT) || a.row_bytes <= 2 * kStepBytes) return launch_thin<DT, YT, GATE>(a, st);
  const int64_t feature_tiles = (a.features + kTiledRows / (GATE ? 2 : 1) - 1) / (kTiledRows / (GATE ? 2 : 1));
  auto cost = [&](int tt) { return tiled_cost(tt, a.rows, a.slots, feature_tiles, p.cus); };
  const float one = cost(1), two = cost(2), four = cost(4);
  if constexpr (tiled_large(DT))
    if (four <= one && four <= two) return launch_tiled<DT, YT, GATE, 4>(a, p.cus, st);
  return one <= two ? launch_tiled<DT, YT, GATE, 1>(a, p.cus, st) : launch_tiled<DT, YT, GATE, 2>(a, p.cus, st);
}

// call(x_dtype, y_dtype, gate), as constants, for a shape that eep_product_create accepts.
template <int N>
using Const = std::integral_constant<int, N>;
template <class Call>
hipError_t with_types(const eep_product_config& f, Call call) {
  const auto with_x = [&](auto x) {
    if (f.gate == EEP_GATE_SILU) {
      const std::true_type gate;
      if (f.y_dtype == EEP_FP8_E4M3) return call(x, Const<EEP_FP8_E4M3>(), gate);
      return f.y_dtype == EEP_BF16 ? call(x, Const<EEP_BF16>(), gate) : call(x, Const<EEP_F32>(), gate);
    }
    const std::false_type gate;
    return f.y_dtype == EEP_BF16 ? call(x, Const<EEP_BF16>(), gate) : call(x, Const<EEP_F32>(), gate);
  };
  if (f.x_dtype == EEP_FP8_E4M3) return with_x(Const<EEP_FP8_E4M3>());
  return f.x_dtype == EEP_BF16 ? with_x(Const<EEP_BF16>()) : with_x(Const<EEP_F32>());
}

}  // namespace eep

using namespace eep;

extern "C" {

int eep_product_create(const eep_product_config* cfg, eep_product** out) {
  if (!out) return EEP_ERR_INVALID_ARG;
  *out = nullptr;
  if (!cfg) return EEP_ERR_INVALID_ARG;
  const eep_product_config& f = *cfg;
  const bool fp8 = f.x_dtype == EEP_FP8_E4M3, gated = f.gate == EEP_GATE_SILU;
  if (f.num_slots < 1 || f.num_slots > 65536 || f.in_features < 1 || f.out_features < 1 ||
      f.in_features > (1 << 21) || f.out_features > (1 << 21) || f.max_rows < 0 || f.max_rows > (1 << 30))
    return EEP_ERR_INVALID_ARG;
  if ((f.x_dtype != EEP_F32 && f.x_dtype != EEP_BF16 && !fp8) ||
      (f.y_dtype != EEP_F32 && f.y_dtype != EEP_BF16 && f.y_dtype != EEP_FP8_E4M3) ||
      (!gated && f.gate != EEP_GATE_NONE) || (f.y_dtype == EEP_FP8_E4M3 && !gated))
    return EEP_ERR_INVALID_ARG;
  const int64_t in_bytes = (int64_t)f.in_features * dtype_bytes(f.x_dtype);
  if (in_bytes % 16 || (int64_t)f.out_features * dtype_bytes(f.y_dtype) % 16) return EEP_ERR_ALIGN;
  if ((fp8 && f.in_features % kScaleBlock != 0) ||
      ((f.y_dtype == EEP_FP8_E4M3 || (fp8 && gated)) && f.out_features % kScaleBlock != 0))
    return EEP_ERR_INVALID_ARG;
  const int64_t weight_rows = (int64_t)f.out_features * (gated ? 2 : 1);
  const int64_t packed = weight_rows * in_bytes;
  const int64_t packed_scale =
      fp8 ? (weight_rows + kScaleBlock - 1) / kScaleBlock * (f.in_features / kScaleBlock) * (int64_t)sizeof(float) : 0;
  if (f.slot_stride < 0 || f.scale_stride < 0 || (f.slot_stride != 0 && f.slot_stride < packed) ||
      (f.scale_stride != 0 && f.scale_stride < packed_scale))
    return EEP_ERR_INVALID_ARG;
  if (f.slot_stride % 16 || f.scale_stride % 4) return EEP_ERR_ALIGN;
  eep_product* p = new (std::nothrow) eep_product();
  if (!p) return EEP_ERR_INVALID_ARG;
  p->cfg = f;
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess ||
      hipDeviceGetAttribute(&p->cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess ||
      with_types(f, [](auto x_dtype, auto y_dtype, auto gate) {
        return allow_lds<x_dtype.value, y_dtype.value, gate.value>();
      }) != hipSuccess) {
    (void)hipGetLastError();
    delete p;
    return EEP_ERR_HIP;
  }
  if (f.y_dtype == EEP_FP8_E4M3) {
    const int64_t value_bytes = (int64_t)kFewGroups * kThinTokens * kScaleBlock * sizeof(float);
    void* workspace = nullptr;
    hipError_t e = hipMalloc(&workspace, value_bytes + kFewGroups * sizeof(uint32_t));
    if (e == hipSuccess) {
      p->values = (float*)workspace;
      p->arrived = (uint32_t*)((uint8_t*)workspace + value_bytes);
      e = launch_fill((int32_t*)p->arrived, 0, kFewGroups, nullptr);
      if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
      if (e != hipSuccess) (void)hipFree(workspace);
    }
    if (e != hipSuccess) {
      (void)hipGetLastError();
      delete p;
      return EEP_ERR_HIP;
    }
  }
  p->slot_stride = f.slot_stride ? f.slot_stride : packed;
  p->scale_stride = f.scale_stride ? f.scale_stride : packed_scale;
  *out = p;
  return EEP_OK;
}

int eep_product_destroy(eep_product* product) {
  if (!product) return EEP_OK;
  const hipError_t e = hipDeviceSynchronize(), e2 = hipFree(product->values);
  delete product;
  return e == hipSuccess && e2 == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

int eep_expert_product(eep_product* product, const void* x, const float* x_scale, const void* w, const float* w_scale,
                       const int32_t* offset, void* y, float* y_scale, int32_t rows, void* stream) {
  if (!product || rows < 0 || rows > product->cfg.max_rows) return EEP_ERR_INVALID_ARG;
  const eep_product_config& f = product->cfg;
  const bool fp8 = f.x_dtype == EEP_FP8_E4M3;
  if (rows == 0) return EEP_OK;
  if (!x || !w || !y || (x_scale != nullptr) != fp8 || (w_scale != nullptr) != fp8 || (y_scale != nullptr) != (f.y_dtype == EEP_FP8_E4M3) ||
      (offset == nullptr && f.num_slots != 1))
    return EEP_ERR_INVALID_ARG;
  if (((uintptr_t)x & 15u) || ((uintptr_t)w & 15u) || ((uintptr_t)y & 15u) || ((uintptr_t)x_scale & 3u) ||
      ((uintptr_t)w_scale & 3u) || ((uintptr_t)offset & 3u) || ((uintptr_t)y_scale & 3u))
    return EEP_ERR_ALIGN;
  ProductArgs a = {};
  a.x = (const uint8_t*)x;
  a.w = (const uint8_t*)w;
  a.x_scale = x_scale;
  a.w_scale = w_scale;
  a.offset = offset;
  a.y = (uint8_t*)y;
  a.y_scale = y_scale;
  a.rows = rows;
  a.slots = f.num_slots;
  a.row_bytes = f.in_features * dtype_bytes(f.x_dtype);
  a.features = f.out_features;
  a.slot_stride = product->slot_stride;
  a.scale_stride = product->scale_stride;
  const hipError_t e = with_types(f, [&](auto x_dtype, auto y_dtype, auto gate) {
    return launch_product<x_dtype.value, y_dtype.value, gate.value>(*product, a, (hipStream_t)stream);
  });
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

}  // extern "C"
