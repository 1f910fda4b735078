// What stands in front of dispatch in a layer: the residual addition with its norm and 8-bit codes, and the
// router's choice.
#include "eep_internal.hpp"
#include "numbers.hpp"
#include "rows.hpp"

namespace eep {

// ---------------------------------------------------------------------------
// residual norm: h = x + r;  v = h / sqrt(mean(h^2) + eps) * g;  codes of v with a scale per group.
//
// One workgroup has a row, all of it in registers (NV vectors of 8 channels a thread, neighbouring threads on
// neighbouring vectors): the row is read once, and only the sum of squares crosses wavefronts.  The lanes of
// a scale group are neighbours of one wavefront.  Bound by memory at many rows, by one trip to memory and
// the exchange at few.  Measured: 16384 rows of 7168 bf16 with residual, sum, y and codes 177 us (6.0 TB/s; with plain instead of
// non-temporal stores 196, with up to 128 / 256 / 1024 threads a row 196 / 187 / 185); 5976 rows of 2880 fp32 38.9 us (6.2 TB/s);
// one row of 7168 3.4 us on the device.
// ---------------------------------------------------------------------------
constexpr int kNormMaxHidden = 65536;  // 1024 threads of 8 vectors

struct NormArgs {
  const void *x, *residual, *gain;
  void *sum, *y;
  uint8_t* code;
  float* code_scale;
  int H;
  int lanes_per_group;  // 0: no codes
  float epsilon;
};

template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t vec, float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 d = ((const u32x4*)base)[vec];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(d[i]);
      v[2 * i + 1] = bf16_hi(d[i]);
    }
  } else {
    const f32x4 a = ((const f32x4*)base)[2 * vec], b = ((const f32x4*)base)[2 * vec + 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t vec, const float (&v)[8]) {
  if constexpr (BF16) {
    u32x4 d;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    __builtin_nontemporal_store(d, &((u32x4*)base)[vec]);
  } else {
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, &((f32x4*)base)[2 * vec]);
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, &((f32x4*)base)[2 * vec + 1]);
  }
}

// The sum over groups of 16 or all 64 lanes, in every lane.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
  return fold<LANES>(v, [](float a, float b) { return a + b; });
}

template <bool IN_BF16, bool GAIN_BF16, bool OUT_BF16, int NV>
__global__ __launch_bounds__(1024) void k_norm(NormArgs a, int64_t first) {
  __shared__ float s_part[16];
  const int64_t row = first + blockIdx.x;
  const int vecs = a.H / 8, threads = blockDim.x, tid = threadIdx.x;
  const int64_t row_vec = row * vecs;
  float h[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int v = j * threads + tid;
    if (v < vecs) {
      load8<IN_BF16>(a.x, row_vec + v, h[j]);
      if (a.residual != nullptr) {
        float r[8];
        load8<IN_BF16>(a.residual, row_vec + v, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] += r[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = 0.0f;
    }
  }
  auto sum_squares = [&](float by) {
    float squares = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = h[j][i] * by;
        squares = fmaf(v, v, squares);
      }
    }
    squares = lane_sum<64>(squares);
    if (threads > 64) {
      if ((tid & 63) == 0) s_part[tid >> 6] = squares;
      __syncthreads();
      squares = 0.0f;
      for (int w = 0; w < threads / 64; ++w) squares += s_part[w];
    }
    return squares;
  };
  // Squares of finite values may be too large for fp32, or too small: each is cut off at 2^-149, which a mean beside epsilon
  // of 2^-100 does not feel.  The sum of such a row is that of the row times a power of two, epsilon times its square; the row
  // itself is multiplied by the larger of the two factors first, so that no small value of it is lost.
  float by = 1.0f;
  float mean = sum_squares(1.0f) / (float)a.H;
  if (mean == INFINITY || mean + a.epsilon < 0x1p-100f) {
    by = mean == INFINITY ? 0x1p-80f : 0x1p100f;
    __syncthreads();
    mean = sum_squares(by) / (float)a.H;
  }
  const float inv = 1.0f / sqrtf(mean + a.epsilon * by * by);
  const float factor = by > 1.0f ? by : inv, last_factor = by > 1.0f ? inv : by;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int v = j * threads + tid;
    if (v >= vecs) continue;  // (whole groups are in or out)
    if (a.sum != nullptr) store8<IN_BF16>(a.sum, row_vec + v, h[j]);
    float g[8];
    load8<GAIN_BF16>(a.gain, v, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = h[j][i] * factor * last_factor * g[i];
    if (a.y != nullptr) store8<OUT_BF16>(a.y, row_vec + v, h[j]);
    if (a.lanes_per_group != 0) {
      const float scale = scale_of(group_max(top_magnitude<8>(h[j]), a.lanes_per_group));
      if ((tid & (a.lanes_per_group - 1)) == 0)
        a.code_scale[row * (vecs / a.lanes_per_group) + v / a.lanes_per_group] = scale;
      u32x2 c;
      c[0] = codes4(h[j][0], h[j][1], h[j][2], h[j][3], scale);
      c[1] = codes4(h[j][4], h[j][5], h[j][6], h[j][7], scale);
      __builtin_nontemporal_store(c, &((u32x2*)a.code)[row_vec + v]);
    }
  }
}

template <bool IN_BF16, bool GAIN_BF16, bool OUT_BF16>
hipError_t launch_norm(const NormArgs& a, int T, hipStream_t st) {
  const int vecs = a.H / 8;
  // vectors a thread: one at few rows, up to 1024 threads; at many rows up to 512 threads, of which a CU takes more workgroups
  int nv = 1;
  while (nv < 8 && (vecs > nv * 1024 || (T >= 1024 && vecs > nv * 512))) nv *= 2;
  const int threads = ((vecs + nv - 1) / nv + 63) / 64 * 64;
  return in_launches(T, max_blocks(threads), [&](int64_t first, int64_t n) {
    const dim3 grid((unsigned)n), block((unsigned)threads);
    switch (nv) {
      case 1: hipLaunchKernelGGL((k_norm<IN_BF16, GAIN_BF16, OUT_BF16, 1>), grid, block, 0, st, a, first); break;
      case 2: hipLaunchKernelGGL((k_norm<IN_BF16, GAIN_BF16, OUT_BF16, 2>), grid, block, 0, st, a, first); break;
      case 4: hipLaunchKernelGGL((k_norm<IN_BF16, GAIN_BF16, OUT_BF16, 4>), grid, block, 0, st, a, first); break;
      default: hipLaunchKernelGGL((k_norm<IN_BF16, GAIN_BF16, OUT_BF16, 8>), grid, block, 0, st, a, first);
    }
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------------------
// route: the k largest of E logits, ties to the lower index, and their softmax weights.
//
// A group of LANES lanes has a token, lane l of it the logits [l * NV, (l + 1) * NV), so that the order of the indices is the
// order of lanes and of registers.  A round finds the largest of the lanes' best; the first lane that has it writes its index,
// strikes out the first register there and looks for its next best.  The values are compared as integers of the same
// order (order_of); 0 is what may not be chosen.
//
// The rounds are the bound, not memory.  At many tokens four share a wavefront (16 lanes, up to 16 logits each) and the
// instructions of a round, whose exchanges stay within a row of lanes; at few, where a round's latency counts, and beyond
// 256 logits a token has one for itself.  Measured, 256 logits, top-8, a token a wavefront / four, us: 32 tokens 4.1 / 6.0,
// 4096 4.6 / 5.4, 8192 6.5 / 6.0, 128 logits, 16384 tokens 10.7 / 5.7; 16384 tokens of 256 bf16 logits 11.0 / 8.7, with the index in the
// value's free bits 6.9.
// ---------------------------------------------------------------------------
constexpr int kRouteMaxExperts = 4096;
constexpr int kRouteShared = 8192;  // tokens from which four share a wavefront

// An integer that grows with the value; 0 for -infinity and NaN.  -0 and +0 are one value.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (!(v > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
// exp(v - top) where top >= v, also where both are +infinity
__device__ __forceinline__ float exp_below(float v, float top) { return v == top ? 1.0f : expf(v - top); }

// What a round compares.  bf16 logits leave 16 bits for the index, the lower one above: no two are equal, and a round needs no
// search for the first of them.  0: not to be chosen.
template <bool BF16>
__device__ __forceinline__ uint32_t key_of(float v, int index) {
  const uint32_t o = order_of(v);
  if constexpr (!BF16) return o;
  return o != 0 ? (o & 0xffff0000u) | (0xffffu - (uint32_t)index) : 0;
}
template <bool BF16>
__device__ __forceinline__ float value_of_key(uint32_t key) {
  // (the bits that a negative value's order has below the bf16 are ones)
  return value_of(BF16 ? (key & 0x80000000u ? key & 0xffff0000u : key | 0xffffu) : key);
}

// FOURS: four logits at a time, of rows that are whole fours and aligned to them.
template <bool BF16, int LANES, int NV, bool FOURS>
__global__ __launch_bounds__(256) void k_route(const void* __restrict__ logits, int32_t* __restrict__ topk_idx,
                                               float* __restrict__ topk_w, int E, int k, int over_all, int64_t first,
                                               int64_t end) {
  constexpr int kTokens = 256 / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const int64_t t = first + (int64_t)blockIdx.x * kTokens + threadIdx.x / LANES;
  if (t >= end) return;  // (a group's lanes go together)
  uint32_t o[NV];
  if constexpr (FOURS) {
#pragma unroll
    for (int i = 0; i < NV; i += 4) {
      const int e = lane * NV + i;
      float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (e < E) {
        if constexpr (BF16) {
          const u32x2 d = *(const u32x2*)((const uint16_t*)logits + t * E + e);
          v[0] = bf16_lo(d[0]), v[1] = bf16_hi(d[0]), v[2] = bf16_lo(d[1]), v[3] = bf16_hi(d[1]);
        } else {
          const f32x4 d = *(const f32x4*)((const float*)logits + t * E + e);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = d[j];
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i + j] = key_of<BF16>(v[j], e + j);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = lane * NV + i;
      o[i] = 0;
      if (e < E)
        o[i] = key_of<BF16>(BF16 ? __uint_as_float((uint32_t)((const uint16_t*)logits)[t * E + e] << 16)
                                 : ((const float*)logits)[t * E + e], e);
    }
  }
  uint32_t best = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) best = o[i] > best ? o[i] : best;
  const auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  uint32_t mine = 0;  // lane j: the order of the j-th choice
  const uint32_t top = fold<LANES>(best, larger);
  float all = 0.0f;
  if (over_all != 0 && top != 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) all += o[i] != 0 ? exp_below(value_of_key<BF16>(o[i]), value_of_key<BF16>(top)) : 0.0f;
  }
  uint32_t largest = top;
  for (int j = 0; j < k; ++j) {
    if (j > 0) largest = fold<LANES>(best, larger);
    if (lane == j) mine = largest;
    if (largest == 0) {
      if (lane == 0) topk_idx[t * k + j] = -1;
      continue;
    }
    if constexpr (BF16) {
      uint32_t next = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        o[i] = o[i] == largest ? 0 : o[i];
        next = larger(next, o[i]);
      }
      best = next;
      if (lane == 0) topk_idx[t * k + j] = (int32_t)(0xffffu - (largest & 0xffffu));
      continue;
    }
    uint64_t have = __ballot(best == largest);
    if constexpr (LANES < 64) have = (have >> (threadIdx.x & 63 & ~(LANES - 1))) & ((1ull << LANES) - 1);
    if (lane == __builtin_ctzll(have)) {
      uint32_t next = 0;
      int at = -1;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool struck = at < 0 && o[i] == largest;
        at = struck ? i : at;
        o[i] = struck ? 0 : o[i];
        next = larger(next, o[i]);
      }
      best = next;
      topk_idx[t * k + j] = lane * NV + at;
    }
  }
  const float e = mine != 0 ? exp_below(value_of_key<BF16>(mine), value_of_key<BF16>(top)) : 0.0f;
  const float sum = lane_sum<LANES>(over_all != 0 ? all : e);
  if (lane < k) topk_w[t * k + lane] = mine != 0 ? e / sum : 0.0f;
}

template <bool BF16, int LANES, int NV>
hipError_t launch_route(const eep_router_shape& s, const void* logits, int32_t* topk_idx, float* topk_w, int T,
                        hipStream_t st) {
  constexpr int kTokens = 256 / LANES;
  const bool fours = NV >= 4 && s.num_logical % 4 == 0 && (uintptr_t)logits % (4 * dtype_bytes(s.in_dtype)) == 0;
  return in_launches(T, max_blocks(256) * kTokens, [&](int64_t first, int64_t n) {
    const dim3 grid((unsigned)((n + kTokens - 1) / kTokens)), block(256);
    if constexpr (NV >= 4) {
      if (fours) {
        hipLaunchKernelGGL((k_route<BF16, LANES, NV, true>), grid, block, 0, st, logits, topk_idx, topk_w, s.num_logical,
                           s.topk, s.over_all, first, first + n);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((k_route<BF16, LANES, NV, false>), grid, block, 0, st, logits, topk_idx, topk_w, s.num_logical, s.topk,
                       s.over_all, first, first + n);
    return hipGetLastError();
  });
}

template <bool BF16>
hipError_t launch_route(const eep_router_shape& s, const void* logits, int32_t* topk_idx, float* topk_w, int T,
                        hipStream_t st) {
#define EEP_ROUTE(LANES, NV) \
  if (s.num_logical <= LANES * NV && s.topk <= LANES) return launch_route<BF16, LANES, NV>(s, logits, topk_idx, topk_w, T, st);
  if (T >= kRouteShared) {
    EEP_ROUTE(16, 4) EEP_ROUTE(16, 8) EEP_ROUTE(16, 16)
  }
  EEP_ROUTE(64, 1) EEP_ROUTE(64, 2) EEP_ROUTE(64, 4) EEP_ROUTE(64, 8) EEP_ROUTE(64, 16) EEP_ROUTE(64, 64)
#undef EEP_ROUTE
  return hipErrorInvalidValue;
}

bool f32_or_bf16(int dtype) { return dtype == EEP_F32 || dtype == EEP_BF16; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace eep

using namespace eep;

extern "C" {

int eep_residual_norm(const eep_norm_shape* shape, const void* x, const void* residual, const void* gain, void* sum,
                      void* y, void* code, float* code_scale, int32_t T, void* stream) {
  if (!shape || T < 0) return EEP_ERR_INVALID_ARG;
  const eep_norm_shape& s = *shape;
  if (s.hidden < 8 || s.hidden > kNormMaxHidden || !f32_or_bf16(s.in_dtype) || !f32_or_bf16(s.gain_dtype) ||
      !f32_or_bf16(s.out_dtype) || !(s.epsilon >= 0.0f))
    return EEP_ERR_INVALID_ARG;
  if (s.hidden % 8 != 0) return EEP_ERR_ALIGN;
  const int group = s.scale_group;
  if (group != 0 && (group < 16 || group > 512 || (group & (group - 1)) != 0 || s.hidden % group != 0))
    return EEP_ERR_INVALID_ARG;
  if ((code != nullptr) != (code_scale != nullptr) || (code != nullptr && group == 0)) return EEP_ERR_INVALID_ARG;
  if (T == 0) return EEP_OK;
  if (!x || !gain || (!sum && !y && !code)) return EEP_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(gain) || !aligned16(sum) || !aligned16(y) ||
      !aligned16(code) || ((uintptr_t)code_scale & 3u))
    return EEP_ERR_ALIGN;
  const NormArgs a = {x, residual, gain, sum, y, (uint8_t*)code, code_scale, s.hidden, code ? group / 8 : 0, s.epsilon};
  hipStream_t st = (hipStream_t)stream;
  const int kind = (s.in_dtype == EEP_BF16) * 4 + (s.gain_dtype == EEP_BF16) * 2 + (s.out_dtype == EEP_BF16);
  hipError_t e;
  switch (kind) {
    case 0: e = launch_norm<false, false, false>(a, T, st); break;
    case 1: e = launch_norm<false, false, true>(a, T, st); break;
    case 2: e = launch_norm<false, true, false>(a, T, st); break;
    case 3: e = launch_norm<false, true, true>(a, T, st); break;
    case 4: e = launch_norm<true, false, false>(a, T, st); break;
    case 5: e = launch_norm<true, false, true>(a, T, st); break;
    case 6: e = launch_norm<true, true, false>(a, T, st); break;
    default: e = launch_norm<true, true, true>(a, T, st);
  }
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

int eep_route(const eep_router_shape* shape, const void* logits, int32_t* topk_idx, float* topk_w, int32_t T,
              void* stream) {
  if (!shape || T < 0) return EEP_ERR_INVALID_ARG;
  const eep_router_shape& s = *shape;
  if (s.num_logical < 1 || s.num_logical > kRouteMaxExperts || s.topk < 1 || s.topk > kMaxTopk ||
      s.topk > s.num_logical || !f32_or_bf16(s.in_dtype))
    return EEP_ERR_INVALID_ARG;
  if (T == 0) return EEP_OK;
  if (!logits || !topk_idx || !topk_w) return EEP_ERR_INVALID_ARG;
  if ((uintptr_t)logits % dtype_bytes(s.in_dtype) || ((uintptr_t)topk_idx & 3u) || ((uintptr_t)topk_w & 3u))
    return EEP_ERR_ALIGN;
  const hipError_t e = s.in_dtype == EEP_BF16 ? launch_route<true>(s, logits, topk_idx, topk_w, T, (hipStream_t)stream)
                                              : launch_route<false>(s, logits, topk_idx, topk_w, T, (hipStream_t)stream);
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

}  // extern "C"
