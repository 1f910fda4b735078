// The layer norm, and the gradients of both norms: of their rows, gain and bias.
#include <new>

#include "eep_internal.hpp"
#include "numbers.hpp"

struct eep_norm_grad {
  eep_norm_grad_config cfg;
  int groups;      // rows of partial sums
  float* partial;  // [groups][hidden] of the gain, behind them as many of the bias
};

namespace eep {

constexpr int kNormMaxWidth = 65536;

// Sums over the workgroup of K values, in every thread, always added in the same order.  Successive sums take the two buffers
// in turn, so that one barrier each is enough.
constexpr int kSums = 4;
struct BlockSums {
  float part[2][16][kSums];
};
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], BlockSums& s, int& turn) {
  const int threads = blockDim.x;
#pragma unroll
  for (int i = 0; i < K; ++i) v[i] = lane_sum<64>(v[i]);
  if (threads <= 64) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < K; ++i) s.part[turn][threadIdx.x >> 6][i] = v[i];
  }
  __syncthreads();
  const int w = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < K; ++i) v[i] = lane_sum<16>(w < threads / 64 ? s.part[turn][w][i] : 0.0f);
  turn ^= 1;
}

__device__ __forceinline__ void load8_any(bool bf16, const void* base, int64_t vec, float (&v)[8]) {
  if (bf16)
    load8<true>(base, vec, v);
  else
    load8<false>(base, vec, v);
}

// What a row has to be multiplied with so that its squares fit fp32 (1 for nearly every row), which has been multiplied by `by`: one whose
// sum alone left fp32 goes back to its own size, where epsilon counts.
__device__ __forceinline__ float fitting(float mean_square, float epsilon, float by) {
  if (by == 0x1p-80f) return mean_square < 0x1p-60f ? 0x1p80f : 1.0f;
  if (by != 1.0f) return 1.0f;
  if (!(mean_square < INFINITY)) return 0x1p-80f;
  return mean_square + epsilon < 0x1p-100f ? 0x1p100f : 1.0f;
}

// The mean square of values without their mean, which is small beside them.  (One that left fp32 stays what it is.)
__device__ __forceinline__ float without(float mean_square, float mean) {
  return mean_square < INFINITY ? fmaxf(fmaf(-mean, mean, mean_square), 0.0f) : mean_square;
}

// What is still to be taken out of every value of a centred row: its mean, as roundings left it, where that outweighs what lies around it
// (a row of equal values, mostly, whose mean square would else be a difference of roundings), and wherever the row is scaled.
__device__ __forceinline__ float stray(float left, float mean_square, float epsilon, float by, float more) {
  const bool out = more != 1.0f || left * left > mean_square + epsilon * by * by;
  return out && fabsf(left) < INFINITY ? left : 0.0f;
}
// Times that a row is scaled or centred again: equal values near the largest number take seven, each of which leaves 2^-22 of their
// mean; without that they would go back and forth between two scales, at one of which their squares leave fp32.
constexpr int kRefits = 12;

// ---------------------------------------------------------------------------
// layer norm: h = x + r;  d = h - mean(h);  y = d / sqrt(mean(d^2) + eps) * g + b.
//
// A workgroup has a row, all of it in registers, as the residual norm's kernel does; the mean and the sum of squares are two
// trips through LDS.  Bound by memory at many rows: 5976 rows of 2880 fp32 with residual and sum 40 us (6.0 TB/s).
// ---------------------------------------------------------------------------
struct LayerNormArgs {
  const void *x, *residual, *gain, *bias;
  void *sum, *y;
  int H;
  bool gain_bf16;
  float epsilon;
};

// Takes the mean out of h, but for what roundings leave of it: a row whose sum leaves fp32 is scaled first.  Returns the factor that h
// then holds.
template <int NV>
__device__ __forceinline__ float centre(float (&h)[NV][8], int H, int vecs, BlockSums& s, int& turn) {
  const int threads = blockDim.x, tid = threadIdx.x;
  float by = 1.0f;
  float sum[1] = {0.0f};
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[0] += h[j][i];
  block_sum(sum, s, turn);
  if (!(fabsf(sum[0]) < INFINITY)) {
    by = 0x1p-80f;
    sum[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[j][i] *= by;
        sum[0] += h[j][i];
      }
    block_sum(sum, s, turn);
  }
  const float mean = sum[0] / (float)H;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (j * threads + tid >= vecs) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] -= mean;
  }
  return by;
}

template <bool IN_BF16, bool OUT_BF16, int NV>
__global__ __launch_bounds__(1024) void k_layer_norm(LayerNormArgs a, int64_t first) {
  __shared__ BlockSums s_sums;
  int turn = 0;
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
      if (a.sum != nullptr) store8<IN_BF16>(a.sum, row_vec + v, h[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = 0.0f;
    }
  }
  float by = centre<NV>(h, a.H, vecs, s_sums, turn);
  float left, mean;  // what is left of the mean, and the mean square without it
  auto mean_square = [&]() {
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[0] += h[j][i];
        sum[1] = fmaf(h[j][i], h[j][i], sum[1]);
      }
    block_sum(sum, s_sums, turn);
    left = sum[0] / (float)a.H;
    mean = without(sum[1] / (float)a.H, left);
  };
  mean_square();
  for (int fit = 0; fit < kRefits; ++fit) {
    const float more = fitting(mean, a.epsilon, by), off = stray(left, mean, a.epsilon, by, more);
    if (more == 1.0f && off == 0.0f) break;
    by *= more;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * threads + tid >= vecs) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = (h[j][i] - off) * more;
    }
    mean_square();
  }
  const float inv = 1.0f / sqrtf(mean + a.epsilon * by * by);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int v = j * threads + tid;
    if (v >= vecs) continue;
    float g[8], b[8];
    load8_any(a.gain_bf16, a.gain, v, g);
    if (a.bias != nullptr)
      load8_any(a.gain_bf16, a.bias, v, b);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = fmaf((h[j][i] - left) * inv, g[i], b[i]);
    store8<OUT_BF16>(a.y, row_vec + v, h[j]);
  }
}

template <bool IN_BF16, bool OUT_BF16>
static hipError_t launch_layer_norm(const LayerNormArgs& a, int T, hipStream_t st) {
  const int vecs = a.H / 8;
  int nv = 1;  // vectors a thread, as the residual norm has them
  while (nv < 8 && (vecs > nv * 1024 || (T >= 1024 && vecs > nv * 512))) nv *= 2;
  const int threads = ((vecs + nv - 1) / nv + 63) / 64 * 64;
  return in_launches(T, max_blocks(threads), [&](int64_t first, int64_t n) {
    const dim3 grid((unsigned)n), block((unsigned)threads);
    switch (nv) {
      case 1: hipLaunchKernelGGL((k_layer_norm<IN_BF16, OUT_BF16, 1>), grid, block, 0, st, a, first); break;
      case 2: hipLaunchKernelGGL((k_layer_norm<IN_BF16, OUT_BF16, 2>), grid, block, 0, st, a, first); break;
      case 4: hipLaunchKernelGGL((k_layer_norm<IN_BF16, OUT_BF16, 4>), grid, block, 0, st, a, first); break;
      default: hipLaunchKernelGGL((k_layer_norm<IN_BF16, OUT_BF16, 8>), grid, block, 0, st, a, first);
    }
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------------------
// the norms' gradients: with d = h (or h - mean(h)), u = d / sqrt(mean(d^2) + eps), v = grad_y * gain,
//   grad_h = (v - u * mean(v * u) [- mean(v)]) / sqrt(mean(d^2) + eps) + grad_sum,
//   grad_gain = the sum over rows of grad_y * u, grad_bias = that of grad_y.
//
// A workgroup goes over every so manieth row; a thread has the same channels of each, whose gain and bias sums stay in its
// registers, and the next row's loads are under way while this one's sums cross the workgroup.  The sums of the workgroups
// are left in the workspace and added up, in their order, by a second kernel.  Bound by memory: 16384 rows of 7168 bf16 with grad_sum 159 to 174 us
// (5.4 to 5.9 TB/s; with four exchanges a row, the gain from memory and one workgroup to a CU 242; 1 / 4 / 8 workgroups a CU 233 / 165 / 192; up
// to 1024 / 256 threads 167 / 257; plain stores 170); centred 207 to 219; 64 centred rows 9.6, latency (12.2 with two vectors a thread).
//
// That is so for rows of up to 8192 channels, of which the main variants spill 32 registers a lane at most.  Up to 16384 fp32 rows spill 90 to
// 142: 8192 rows of 16384 bf16 / fp32 4.6 / 3.0 TB/s (centred 3.9 / 2.8).  Above that neither the sums nor the next row fit: 738 to
// 1285 registers a lane are spilled, 1.5 to 1.9 KB, and every row goes through scratch memory: 4096 rows of 16392 0.7 / 0.8 TB/s, 2048
// of 65536 0.7 / 0.95 (centred 0.55 / 0.8 and 0.65 / 0.9).
// ---------------------------------------------------------------------------
struct NormGradArgs {
  const void *h, *gain, *grad_y, *grad_sum;
  void* grad_h;
  float* partial;  // [gridDim.x][H], behind gridDim.x of them those of the bias; NULL: none wanted
  int H, T;
  bool gain_bf16;
  float epsilon;
};

template <bool BF16>
struct Raw8 {
  u32x4 d[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* base, int64_t vec) {
    const u32x4* from = (const u32x4*)base + vec * (BF16 ? 1 : 2);
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) d[i] = __builtin_nontemporal_load(from + i);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (BF16)
      return i & 1 ? bf16_hi(d[0][i >> 1]) : bf16_lo(d[0][i >> 1]);
    else
      return __uint_as_float(d[i >> 2][i & 3]);
  }
};

// Workgroups to a CU: as many as registers allow; the rows of fp32 inputs are twice as many bytes under way.
constexpr int norm_grad_threads(int nv) { return nv == 8 || nv == 1 ? 1024 : 512; }
constexpr int norm_grad_waves(bool in_bf16, int nv) { return nv == 8 || nv == 1 || (in_bf16 && nv <= 2) ? 4 : 2; }

template <bool IN_BF16, bool OUT_BF16, bool CENTRED, int NV>
__global__ __launch_bounds__(norm_grad_threads(NV), norm_grad_waves(IN_BF16, NV)) void k_norm_grad(NormGradArgs a) {
  __shared__ BlockSums s_sums;
  extern __shared__ f32x4 s_gain[];  // of rows that fit it
  constexpr bool kGainInLds = NV <= 2;
  const int vecs = a.H / 8, threads = blockDim.x, tid = threadIdx.x;
  const float count = (float)a.H;
  int turn = 0;
  Raw8<IN_BF16> h_raw[NV], stream_raw[NV];
  Raw8<OUT_BF16> grad_raw[NV];
  float gain_sum[NV][8], bias_sum[CENTRED ? NV : 1][8];
  const auto fetch = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int v = j * threads + tid;
      if (v >= vecs) continue;
      h_raw[j].load(a.h, row * vecs + v);
      grad_raw[j].load(a.grad_y, row * vecs + v);
      if (a.grad_sum != nullptr) stream_raw[j].load(a.grad_sum, row * vecs + v);
    }
  };
  const auto gain_of = [&](int j, float (&g)[8]) {
    const int at = j * threads + tid;
    if constexpr (kGainInLds) {
      const f32x4 low = s_gain[2 * at], high = s_gain[2 * at + 1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g[i] = low[i];
        g[4 + i] = high[i];
      }
    } else {
      load8_any(a.gain_bf16, a.gain, at, g);
    }
  };
  fetch(blockIdx.x);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = j * threads + tid;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      gain_sum[j][i] = 0.0f;
      if constexpr (CENTRED) bias_sum[j][i] = 0.0f;
    }
    if (kGainInLds && at < vecs) {
      float g[8];
      load8_any(a.gain_bf16, a.gain, at, g);
      // (every thread reads what it wrote itself)
      s_gain[2 * at] = f32x4{g[0], g[1], g[2], g[3]};
      s_gain[2 * at + 1] = f32x4{g[4], g[5], g[6], g[7]};
    }
  }
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    float d[NV][8];
    Raw8<IN_BF16> stream[NV];
    Raw8<OUT_BF16> grad[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const bool in = j * threads + tid < vecs;
#pragma unroll
      for (int i = 0; i < 8; ++i) d[j][i] = in ? h_raw[j].at(i) : 0.0f;
      stream[j] = stream_raw[j];
      grad[j] = grad_raw[j];
    }
    if (row + gridDim.x < a.T) fetch(row + gridDim.x);
    float by = 1.0f;
    if constexpr (CENTRED) by = centre<NV>(d, a.H, vecs, s_sums, turn);
    // of d * d and v * d; centred, of d, which roundings have left, and of v
    constexpr int kOfV = CENTRED ? 3 : 0;
    float sum[CENTRED ? 4 : 2];
    const auto sums = [&]() {
#pragma unroll
      for (float& v : sum) v = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j * threads + tid >= vecs) continue;
        float g[8];
        gain_of(j, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = grad[j].at(i) * g[i];
          sum[0] = fmaf(d[j][i], d[j][i], sum[0]);
          sum[1] = fmaf(v, d[j][i], sum[1]);
          if constexpr (CENTRED) {
            sum[2] += d[j][i];
            sum[kOfV] += v;
          }
        }
      }
      block_sum(sum, s_sums, turn);
    };
    const auto mean_square = [&]() {
      if constexpr (CENTRED) {
        return without(sum[0] / count, sum[2] / count);
      } else {
        return sum[0] / count;
      }
    };
    sums();
    if constexpr (CENTRED) {
      for (int fit = 0; fit < kRefits; ++fit) {
        const float more = fitting(mean_square(), a.epsilon, by), off = stray(sum[2] / count, mean_square(), a.epsilon, by, more);
        if (more == 1.0f && off == 0.0f) break;
        by *= more;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) d[j][i] = (d[j][i] - off) * more;  // (what lies past the row is used nowhere)
        sums();
      }
    } else {
      // (once or not at all: squares that leave fp32 have a mean of 2^-48 at least times 2^-160.  Counted as above, 173 us for 162.)
      for (float more; (more = fitting(mean_square(), a.epsilon, by)) != 1.0f;) {
        by *= more;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) d[j][i] *= more;
        sums();
      }
    }
    const float inv = 1.0f / sqrtf(mean_square() + a.epsilon * by * by);
    float left = 0.0f, mean = 0.0f;
    if constexpr (CENTRED) {
      left = sum[2] / count;
      mean = sum[kOfV] / count;
    }
    float along = fmaf(-left, mean, sum[1] / count) * inv;  // mean(v * u)
    // Where products of v and d leave fp32, on either side, those of v and u may not; nor has v to leave it where its sum does.
    const bool within = fabsf(sum[1]) < INFINITY && (!CENTRED || fabsf(sum[kOfV]) < INFINITY);
    if (__builtin_expect(!within || (sum[1] != 0.0f && fabsf(sum[1]) < 0x1p-100f), 0)) {
      const float fits = within ? 1.0f : 0x1p-32f;
      float again[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j * threads + tid >= vecs) continue;
        float g[8];
        gain_of(j, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = grad[j].at(i) * g[i] * fits;
          again[0] = fmaf(v, (d[j][i] - left) * inv, again[0]);
          again[1] += v;
        }
      }
      block_sum(again, s_sums, turn);
      along = again[0] / count / fits;
      if constexpr (CENTRED) mean = again[1] / count / fits;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * threads + tid;
      if (at >= vecs) continue;
      float g[8], o[8];
      gain_of(j, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = (d[j][i] - left) * inv, dy = grad[j].at(i);
        gain_sum[j][i] = fmaf(dy, u, gain_sum[j][i]);
        if constexpr (CENTRED) bias_sum[j][i] += dy;
        o[i] = (fmaf(-u, along, dy * g[i]) - mean) * inv * by;
        if (a.grad_sum != nullptr) o[i] += stream[j].at(i);
      }
      if (a.grad_h != nullptr) store8<IN_BF16>(a.grad_h, row * vecs + at, o);
    }
  }
  if (a.partial == nullptr) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = j * threads + tid;
    if (at >= vecs) continue;
    f32x4* to = (f32x4*)(a.partial + (int64_t)blockIdx.x * a.H) + 2 * at;
    to[0] = f32x4{gain_sum[j][0], gain_sum[j][1], gain_sum[j][2], gain_sum[j][3]};
    to[1] = f32x4{gain_sum[j][4], gain_sum[j][5], gain_sum[j][6], gain_sum[j][7]};
    if constexpr (CENTRED) {
      f32x4* bias_to = to + (int64_t)gridDim.x * a.H / 4;
      bias_to[0] = f32x4{bias_sum[j][0], bias_sum[j][1], bias_sum[j][2], bias_sum[j][3]};
      bias_to[1] = f32x4{bias_sum[j][4], bias_sum[j][5], bias_sum[j][6], bias_sum[j][7]};
    }
  }
}

// The sums of the workgroups, column by column; 64 columns and 16 runs of rows a workgroup.
constexpr int kColumnRuns = 16;
__global__ __launch_bounds__(64 * kColumnRuns) void k_norm_columns(const float* partial, float* grad_gain, float* grad_bias, int H,
                                                                   int groups, int accumulate) {
  __shared__ float s_sum[kColumnRuns][64];
  const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
  const int column = blockIdx.x * 64 + lane;
  const bool bias = blockIdx.y != 0;
  float* to = bias ? grad_bias : grad_gain;
  const float* from = partial + (bias ? (int64_t)groups * H : 0);
  float sum = 0.0f;
  if (column < H) {
    const int end = (int)((int64_t)groups * (run + 1) / kColumnRuns);
#pragma unroll 8
    for (int g = (int)((int64_t)groups * run / kColumnRuns); g < end; ++g) sum += from[(int64_t)g * H + column];
  }
  s_sum[run][lane] = sum;
  __syncthreads();
  if (run != 0 || column >= H || to == nullptr) return;
  for (int r = 1; r < kColumnRuns; ++r) sum += s_sum[r][lane];
  to[column] = accumulate != 0 ? to[column] + sum : sum;
}

template <bool IN_BF16, bool OUT_BF16, bool CENTRED>
static hipError_t launch_norm_grad(const NormGradArgs& a, int groups, int most_groups, hipStream_t st) {
  const int vecs = a.H / 8;
  int nv = 1;  // vectors a thread: one where rows are fewer than CUs and latency counts, else so many that threads are up to 512
  if (a.T > most_groups / 2 || vecs > 1024)
    while (nv < 8 && vecs > nv * 512) nv *= 2;
  const dim3 grid((unsigned)groups), block((unsigned)(((vecs + nv - 1) / nv + 63) / 64 * 64));
  const size_t lds = nv <= 2 ? (size_t)a.H * sizeof(float) : 0;
  switch (nv) {
    case 1: hipLaunchKernelGGL((k_norm_grad<IN_BF16, OUT_BF16, CENTRED, 1>), grid, block, lds, st, a); break;
    case 2: hipLaunchKernelGGL((k_norm_grad<IN_BF16, OUT_BF16, CENTRED, 2>), grid, block, lds, st, a); break;
    case 4: hipLaunchKernelGGL((k_norm_grad<IN_BF16, OUT_BF16, CENTRED, 4>), grid, block, lds, st, a); break;
    default: hipLaunchKernelGGL((k_norm_grad<IN_BF16, OUT_BF16, CENTRED, 8>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace eep

using namespace eep;

extern "C" {

int eep_layer_norm(const eep_norm_shape* shape, const void* x, const void* residual, const void* gain, const void* bias, void* sum,
                   void* y, int32_t T, void* stream) {
  if (!shape || T < 0) return EEP_ERR_INVALID_ARG;
  const eep_norm_shape& s = *shape;
  if (s.hidden < 8 || s.hidden > kNormMaxWidth || !f32_or_bf16(s.in_dtype) || !f32_or_bf16(s.gain_dtype) ||
      !f32_or_bf16(s.out_dtype) || s.scale_group != 0 || !(s.epsilon >= 0.0f))
    return EEP_ERR_INVALID_ARG;
  if (s.hidden % 8 != 0) return EEP_ERR_ALIGN;
  if (T == 0) return EEP_OK;
  if (!x || !gain || !y) return EEP_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(gain) || !aligned16(bias) || !aligned16(sum) || !aligned16(y)) return EEP_ERR_ALIGN;
  const LayerNormArgs a = {x, residual, gain, bias, sum, y, s.hidden, s.gain_dtype == EEP_BF16, s.epsilon};
  hipStream_t st = (hipStream_t)stream;
  const bool in = s.in_dtype == EEP_BF16, out = s.out_dtype == EEP_BF16;
  const hipError_t e = in ? (out ? launch_layer_norm<true, true>(a, T, st) : launch_layer_norm<true, false>(a, T, st))
                          : (out ? launch_layer_norm<false, true>(a, T, st) : launch_layer_norm<false, false>(a, T, st));
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

int eep_norm_grad_create(const eep_norm_grad_config* cfg, eep_norm_grad** out) {
  if (!out) return EEP_ERR_INVALID_ARG;
  *out = nullptr;
  if (!cfg) return EEP_ERR_INVALID_ARG;
  const eep_norm_grad_config& f = *cfg;
  if (f.hidden < 8 || f.hidden > kNormMaxWidth || !f32_or_bf16(f.in_dtype) || !f32_or_bf16(f.gain_dtype) ||
      !f32_or_bf16(f.out_dtype) || (f.centred != 0 && f.centred != 1) || !(f.epsilon >= 0.0f))
    return EEP_ERR_INVALID_ARG;
  if (f.hidden % 8 != 0) return EEP_ERR_ALIGN;
  eep_norm_grad* g = new (std::nothrow) eep_norm_grad();
  if (!g) return EEP_ERR_INVALID_ARG;
  g->cfg = f;
  int device = 0, cus = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
  g->groups = 2 * cus;
  if (e == hipSuccess)
    e = hipMalloc((void**)&g->partial, (size_t)g->groups * f.hidden * sizeof(float) * (f.centred ? 2 : 1));
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete g;
    return EEP_ERR_HIP;
  }
  *out = g;
  return EEP_OK;
}

int eep_norm_grad_destroy(eep_norm_grad* grad) {
  if (!grad) return EEP_OK;
  const hipError_t e = hipDeviceSynchronize(), e2 = hipFree(grad->partial);
  delete grad;
  return e == hipSuccess && e2 == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

int eep_norm_grad_run(eep_norm_grad* grad, const void* h, const void* gain, const void* grad_y, const void* grad_sum, void* grad_h,
                      float* grad_gain, float* grad_bias, int32_t accumulate, int32_t T, void* stream) {
  if (!grad || T < 0 || (accumulate != 0 && accumulate != 1)) return EEP_ERR_INVALID_ARG;
  const eep_norm_grad_config& f = grad->cfg;
  if ((grad_bias != nullptr && !f.centred) || (!grad_h && !grad_gain && !grad_bias) || (grad_sum != nullptr && grad_h == nullptr))
    return EEP_ERR_INVALID_ARG;
  if (T > 0 && (!h || !gain || !grad_y)) return EEP_ERR_INVALID_ARG;
  if (!aligned16(h) || !aligned16(gain) || !aligned16(grad_y) || !aligned16(grad_sum) || !aligned16(grad_h) || ((uintptr_t)grad_gain & 3u) ||
      ((uintptr_t)grad_bias & 3u))
    return EEP_ERR_ALIGN;
  hipStream_t st = (hipStream_t)stream;
  const bool columns = grad_gain != nullptr || grad_bias != nullptr;
  const int groups = T < grad->groups ? T : grad->groups;
  const NormGradArgs a = {h, gain, grad_y, grad_sum, grad_h, columns ? grad->partial : nullptr, f.hidden, T, f.gain_dtype == EEP_BF16,
                          f.epsilon};
  hipError_t e = hipSuccess;
  if (T > 0) {
    switch ((f.in_dtype == EEP_BF16) * 4 + (f.out_dtype == EEP_BF16) * 2 + f.centred) {
      case 0: e = launch_norm_grad<false, false, false>(a, groups, grad->groups, st); break;
      case 1: e = launch_norm_grad<false, false, true>(a, groups, grad->groups, st); break;
      case 2: e = launch_norm_grad<false, true, false>(a, groups, grad->groups, st); break;
      case 3: e = launch_norm_grad<false, true, true>(a, groups, grad->groups, st); break;
      case 4: e = launch_norm_grad<true, false, false>(a, groups, grad->groups, st); break;
      case 5: e = launch_norm_grad<true, false, true>(a, groups, grad->groups, st); break;
      case 6: e = launch_norm_grad<true, true, false>(a, groups, grad->groups, st); break;
      default: e = launch_norm_grad<true, true, true>(a, groups, grad->groups, st);
    }
  }
  if (e == hipSuccess && columns) {  // (of no rows: zeros)
    hipLaunchKernelGGL(k_norm_columns, dim3((unsigned)(f.hidden + 63) / 64, f.centred ? 2 : 1), dim3(64 * kColumnRuns), 0, st,
                       grad->partial, grad_gain, grad_bias, f.hidden, groups, accumulate);
    e = hipGetLastError();
  }
  return e == hipSuccess ? EEP_OK : EEP_ERR_HIP;
}

}  // extern "C"
