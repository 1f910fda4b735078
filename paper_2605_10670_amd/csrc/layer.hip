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
// the exchange at few.
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
    ((u32x4*)base)[vec] = d;
  } else {
    ((f32x4*)base)[2 * vec] = f32x4{v[0], v[1], v[2], v[3]};
    ((f32x4*)base)[2 * vec + 1] = f32x4{v[4], v[5], v[6], v[7]};
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
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
    squares = wave_sum(squares);
    if (threads > 64) {
      if ((tid & 63) == 0) s_part[tid >> 6] = squares;
      __syncthreads();
      squares = 0.0f;
      for (int w = 0; w < threads / 64; ++w) squares += s_part[w];
    }
    return squares;
  };
  const float squares = sum_squares(1.0f);
  float inv = 1.0f / sqrtf(squares / (float)a.H + a.epsilon);
  if (squares == INFINITY) {
    // the squares of finite values may be too large for their type; then epsilon is nothing beside them
    __syncthreads();
    inv = 0x1p-80f / sqrtf(sum_squares(0x1p-80f) / (float)a.H);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int v = j * threads + tid;
    if (v >= vecs) continue;  // (whole groups are in or out)
    if (a.sum != nullptr) store8<IN_BF16>(a.sum, row_vec + v, h[j]);
    float g[8];
    load8<GAIN_BF16>(a.gain, v, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = h[j][i] * inv * g[i];
    if (a.y != nullptr) store8<OUT_BF16>(a.y, row_vec + v, h[j]);
    if (a.lanes_per_group != 0) {
      const float scale = scale_of(group_max(top_magnitude<8>(h[j]), a.lanes_per_group));
      if ((tid & (a.lanes_per_group - 1)) == 0)
        a.code_scale[row * (vecs / a.lanes_per_group) + v / a.lanes_per_group] = scale;
      u32x2 c;
      c[0] = codes4(h[j][0], h[j][1], h[j][2], h[j][3], scale);
      c[1] = codes4(h[j][4], h[j][5], h[j][6], h[j][7], scale);
      ((u32x2*)a.code)[row_vec + v] = c;
    }
  }
}

template <bool IN_BF16, bool GAIN_BF16, bool OUT_BF16>
hipError_t launch_norm(const NormArgs& a, int T, hipStream_t st) {
  const int vecs = a.H / 8;
  // vectors a thread: the fewest that fit a workgroup at few rows; at many rows as many as leave two wavefronts
  int nv = 1;
  while (nv < 8 && (vecs > nv * 1024 || (T >= 1024 && vecs > nv * 128))) nv *= 2;
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
// One wavefront has a token, lane l the logits [l * NV, (l + 1) * NV), so that the order of the indices is the order of
// lanes and of registers.  A round finds the largest of the lanes' best, takes the first lane that has it and the
// first register there, and strikes it out.  The values are compared as integers of the same order (order_of);
// 0 is what may not be chosen.
// ---------------------------------------------------------------------------
constexpr int kRouteMaxExperts = 4096;

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

template <bool BF16, int NV>
__global__ __launch_bounds__(256) void k_route(const void* __restrict__ logits, int32_t* __restrict__ topk_idx,
                                               float* __restrict__ topk_w, int E, int k, int over_all, int64_t first,
                                               int64_t end) {
  const int lane = threadIdx.x & 63;
  const int64_t t = first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= end) return;
  uint32_t o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = lane * NV + i;
    o[i] = 0;
    if (e < E)
      o[i] = order_of(BF16 ? __uint_as_float((uint32_t)((const uint16_t*)logits)[t * E + e] << 16)
                           : ((const float*)logits)[t * E + e]);
  }
  uint32_t best = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) best = o[i] > best ? o[i] : best;
  uint32_t mine = 0;  // lane j: the order and the index of the j-th choice
  int32_t choice = -1;
  int32_t index = 0;  // what this lane won last
  uint32_t top = 0;
  float all = 0.0f;
  for (int j = 0; j < k; ++j) {
    const uint32_t largest = group_max(best, 64);
    if (j == 0) {
      top = largest;
      if (over_all != 0 && top != 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) all += o[i] != 0 ? exp_below(value_of(o[i]), value_of(top)) : 0.0f;
      }
    }
    if (largest == 0) break;
    const int winner = __builtin_ctzll(__ballot(best == largest));
    if (lane == winner) {
      // strike out the first register that has it; the next best of what is left
      uint32_t next = 0;
      bool found = false;
      int at = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!found && o[i] == largest) {
          found = true;
          at = i;
          o[i] = 0;
        }
        next = o[i] > next ? o[i] : next;
      }
      best = next;
      index = lane * NV + at;
    }
    const int32_t chosen = __builtin_amdgcn_readlane(index, winner);
    if (lane == j) {
      mine = largest;
      choice = chosen;
    }
  }
  const float e = mine != 0 ? exp_below(value_of(mine), value_of(top)) : 0.0f;
  const float sum = wave_sum(over_all != 0 ? all : e);
  if (lane < k) {
    topk_idx[t * k + lane] = choice;
    topk_w[t * k + lane] = mine != 0 ? e / sum : 0.0f;
  }
}

template <bool BF16>
hipError_t launch_route(const eep_router_shape& s, const void* logits, int32_t* topk_idx, float* topk_w, int T,
                        hipStream_t st) {
  return in_launches(T, max_blocks(256) * 4, [&](int64_t first, int64_t n) {
    const dim3 grid((unsigned)((n + 3) / 4)), block(256);
#define EEP_ROUTE(NV)                                                                                            \
  if (s.num_logical <= 64 * NV) {                                                                                \
    hipLaunchKernelGGL((k_route<BF16, NV>), grid, block, 0, st, logits, topk_idx, topk_w, s.num_logical, s.topk, \
                       s.over_all, first, first + n);                                                            \
    return hipGetLastError();                                                                                    \
  }
    EEP_ROUTE(1) EEP_ROUTE(2) EEP_ROUTE(4) EEP_ROUTE(8) EEP_ROUTE(16) EEP_ROUTE(64)
#undef EEP_ROUTE
    return hipErrorInvalidValue;
  });
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
