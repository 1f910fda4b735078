// The gradients of combine and of dispatch, by the rows that the layout of the forward pass left behind.
#include <type_traits>

#include "eep_internal.hpp"
#include "numbers.hpp"
#include "rows.hpp"

namespace eep {

// N neighbouring values (4 fp32, or 8 of either type) as they lie in memory, and as fp32.
template <bool BF16, int N>
struct Piece {
  u32x4 d[BF16 ? 1 : N / 4];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const u32x4* from = (const u32x4*)base + at * (BF16 ? 1 : N / 4);
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : N / 4); ++i) d[i] = __builtin_nontemporal_load(from + i);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (BF16)
      return i & 1 ? bf16_hi(d[0][i >> 1]) : bf16_lo(d[0][i >> 1]);
    else
      return __uint_as_float(d[i >> 2][i & 3]);
  }
  __device__ __forceinline__ void round(const float (&v)[N]) {
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) d[0][i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i >> 2][i & 3] = __float_as_uint(v[i]);
    }
  }
  // through: as receive rows are stored (rows.hpp), else non-temporal
  __device__ __forceinline__ void store(void* base, int64_t at, bool through) const {
    u32x4* to = (u32x4*)base + at * (BF16 ? 1 : N / 4);
    if (through) {
#pragma unroll
      for (int i = 0; i < (BF16 ? 1 : N / 4); ++i) store_row(to + i, d[i]);
    } else {
#pragma unroll
      for (int i = 0; i < (BF16 ? 1 : N / 4); ++i) __builtin_nontemporal_store(d[i], to + i);
    }
  }
};

struct CombineGradArgs {
  const int32_t *row_of, *slot_of, *src_of, *offset;
  const void *grad_out, *y;
  const float* topk_w;
  void* grad_y;
  float* grad_w;
  int k, pieces;  // of N values, of a row
  bool through;   // how rows are stored
};

// The row of a pair that lost its row_of entry when failure detection dropped its rank within the step (-1: it never had
// one).  A slot's rows are in the order of their pairs.
__device__ __forceinline__ int row_of_dropped(const CombineGradArgs& a, int64_t pair) {
  const int slot = a.slot_of[pair];
  if (slot < 0) return -1;
  int lo = a.offset[slot], hi = a.offset[slot + 1];
  while (lo < hi) {
    const int mid = (lo + hi) / 2, at = a.src_of[mid];
    if (at == pair) return mid;
    if (at < pair)
      lo = mid + 1;
    else
      hi = mid;
  }
  return -1;
}

// ---------------------------------------------------------------------------
// combine's gradient: grad_y[row_of[t, j]] = w[t, j] * grad_out[t], grad_w[t, j] = <grad_out[t], y[row_of[t, j]]>.
//
// A workgroup has B pairs of one token: it reads the token's gradient once for them, and of every pair the row of y, from which
// the products are summed, and writes the row of grad_y beside it.  Bound by memory at many tokens, by one trip and the
// sum across wavefronts at few.  Measured on buffers that are used again and again, 5976 tokens of 2880, top-6, rows bf16, tokens fp32 /
// 16384 of 7168, top-8 / 512 / 128 of them, us: non-temporal stores 92.0 / 813 / 24.9 / 10.4, write-through 82.6 / 815 / 20.9 / 9.2, plain
// 81.7 / 847 / 23.5 / 10.6; on other buffers every time, where the large caches have none of them, 5976 tokens 92 (5.1 TB/s) / 95 / 98.
// Up to 4 / 2 pairs a workgroup (non-temporal) 101 / 888 / 24.8 / 10.4 and 111 / 1034 / 24.9 / 10.3; 256 / 128 threads 92.9 / 816 / 25.1 / 10.6
// and 94.2 / 822 / 26.6 / 10.5.
// ---------------------------------------------------------------------------
constexpr int64_t kThroughBytes = 128 << 20;  // of grad_y, half of what the memory-side cache holds

template <bool Y_BF16, bool OUT_BF16, int N, int B>
__global__ __launch_bounds__(1024) void k_combine_grad(CombineGradArgs a, int64_t first, int batches) {
  __shared__ float s_part[16][B];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int batch = batches > 1 ? blockIdx.x % (unsigned)batches : 0;
  const int64_t t = first + (batches > 1 ? blockIdx.x / (unsigned)batches : blockIdx.x);
  const int j0 = batch * B;
  int row[B];
  float w[B], sum[B];
  uint32_t dropped = 0;
#pragma unroll
  for (int j = 0; j < B; ++j) row[j] = j0 + j < a.k ? a.row_of[t * a.k + j0 + j] : -1;
#pragma unroll
  for (int j = 0; j < B; ++j) {
    sum[j] = 0.0f;
    w[j] = j0 + j < a.k && a.grad_y != nullptr ? a.topk_w[t * a.k + j0 + j] : 0.0f;
  }
#pragma unroll
  for (int j = 0; j < B; ++j)
    if (__builtin_expect(row[j] < 0 && j0 + j < a.k, 0)) {
      // (its row takes part in the experts' gradients and has to be zeros)
      row[j] = row_of_dropped(a, t * a.k + j0 + j);
      if (row[j] >= 0) dropped |= 1u << j;
    }
  for (int v = tid; v < a.pieces; v += threads) {
    Piece<OUT_BF16, N> g;
    Piece<Y_BF16, N> y[B];
    g.load(a.grad_out, t * a.pieces + v);
    if (a.grad_w != nullptr) {
      // (a pair without a row, or a dropped one, loads some row, and its sum is not used)
#pragma unroll
      for (int j = 0; j < B; ++j) y[j].load(a.y, (int64_t)(row[j] >= 0 ? row[j] : 0) * a.pieces + v);
#pragma unroll
      for (int j = 0; j < B; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[j] = fmaf(g.at(i), y[j].at(i), sum[j]);
    }
    if (a.grad_y != nullptr) {
#pragma unroll
      for (int j = 0; j < B; ++j)
        if (row[j] >= 0) {
          float o[N];
          const bool zeros = (dropped >> j) & 1;
#pragma unroll
          for (int i = 0; i < N; ++i) o[i] = zeros ? 0.0f : w[j] * g.at(i);
          Piece<Y_BF16, N> piece;
          piece.round(o);
          piece.store(a.grad_y, (int64_t)row[j] * a.pieces + v, a.through);
        }
    }
  }
  if (a.grad_w == nullptr) return;
#pragma unroll
  for (int j = 0; j < B; ++j) {
    sum[j] = lane_sum<64>(sum[j]);
    if ((tid & 63) == 0) s_part[tid >> 6][j] = sum[j];
  }
  __syncthreads();
  if (tid < B && j0 + tid < a.k) {
    float all = 0.0f;
    for (int i = 0; i < threads / 64; ++i) all += s_part[i][tid];
    bool summed = false;
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (j == tid) summed = row[j] >= 0 && !((dropped >> j) & 1);
    a.grad_w[t * a.k + j0 + tid] = summed ? all : 0.0f;
  }
}

template <bool Y_BF16, bool OUT_BF16, int N>
static hipError_t launch_combine_grad_t(const CombineGradArgs& a, int T, hipStream_t st) {
  // pairs a workgroup: as many as leave a thousand workgroups, up to 8, the batches of a token alike
  const int64_t pairs = (int64_t)T * a.k;
  const int most = pairs < 2 * 1024 ? 1 : pairs < 8 * 1024 ? (int)(pairs / 1024) : 8;
  const int batches = (a.k + most - 1) / most, size = (a.k + batches - 1) / batches;
  // threads: all of a row at a time where workgroups are few, else up to 512
  const int limit = pairs < 2 * 1024 ? 1024 : 512, rounds = (a.pieces + limit - 1) / limit;
  const int threads = ((a.pieces + rounds - 1) / rounds + 63) / 64 * 64;
  return in_launches(T, max_blocks(threads) / batches, [&](int64_t first, int64_t n) {
    const dim3 grid((unsigned)(n * batches)), block((unsigned)threads);
    switch (size) {
#define EEP_PAIRS(B) \
  case B: hipLaunchKernelGGL((k_combine_grad<Y_BF16, OUT_BF16, N, B>), grid, block, 0, st, a, first, batches); break;
      EEP_PAIRS(1) EEP_PAIRS(2) EEP_PAIRS(3) EEP_PAIRS(4) EEP_PAIRS(5) EEP_PAIRS(6) EEP_PAIRS(7) EEP_PAIRS(8)
#undef EEP_PAIRS
    }
    return hipGetLastError();
  });
}

hipError_t launch_combine_grad(eep_ctx* c, const void* y, const float* topk_w, const void* grad_out, void* grad_y, float* grad_w,
                               int T, hipStream_t st) {
  CombineGradArgs a = {c->row_of, c->slot_of, c->src_of, c->offset, grad_out, y, topk_w, grad_y, grad_w, c->k, 0, false};
  const bool yb = c->cfg.y_dtype == EEP_BF16, ob = c->cfg.out_dtype == EEP_BF16;
  const int n = yb || ob ? 8 : 4;
  a.pieces = c->H / n;
  a.through = (int64_t)T * c->k * c->y_row_bytes <= kThroughBytes;
  if (yb && ob) return launch_combine_grad_t<true, true, 8>(a, T, st);
  if (yb) return launch_combine_grad_t<true, false, 8>(a, T, st);
  if (ob) return launch_combine_grad_t<false, true, 8>(a, T, st);
  return launch_combine_grad_t<false, false, 4>(a, T, st);
}

// ---------------------------------------------------------------------------
// dispatch's gradient: grad_x[t] = sum over routed j, ascending, of grad_recv[row_of[t, j]]: combine without weights.
//
// As there, a wavefront has 64 pieces of one token's rows, their loads all under way together.  Bound by memory: 16384 tokens of 7168 bf16,
// top-8, 323 us (6.2 TB/s).
// ---------------------------------------------------------------------------
template <bool Y_BF16, bool OUT_BF16, int N>
__global__ __launch_bounds__(64) void k_dispatch_grad(const int32_t* __restrict__ row_of, const void* __restrict__ grad_recv,
                                                      void* __restrict__ grad_x, int k, int pieces, uint32_t parts,
                                                      uint32_t magic, int64_t first_token) {
  const uint32_t n = token_of(blockIdx.x, parts, magic);
  const int v = (int)(blockIdx.x - n * parts) * 64 + threadIdx.x;
  const int64_t t = first_token + n;
  if (v >= pieces) return;
  const int32_t* rows = row_of + t * k;
  float acc[N] = {};
  const auto batch = [&](auto size, int j0) {
    constexpr int B = decltype(size)::value;
    int row[B];
    Piece<Y_BF16, N> d[B];
#pragma unroll
    for (int j = 0; j < B; ++j) row[j] = rows[j0 + j];
    // (a pair without a row loads row 0, and its term is left out)
#pragma unroll
    for (int j = 0; j < B; ++j) d[j].load(grad_recv, (int64_t)(row[j] >= 0 ? row[j] : 0) * pieces + v);
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (row[j] >= 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += d[j].at(i);
      }
  };
  int j = 0;
  for (; j + 8 <= k; j += 8) batch(std::integral_constant<int, 8>(), j);
  if (j + 4 <= k) {
    batch(std::integral_constant<int, 4>(), j);
    j += 4;
  }
  if (j + 2 <= k) {
    batch(std::integral_constant<int, 2>(), j);
    j += 2;
  }
  if (j < k) batch(std::integral_constant<int, 1>(), j);
  Piece<OUT_BF16, N> piece;
  piece.round(acc);
  piece.store(grad_x, t * pieces + v, false);
}

template <bool Y_BF16, bool OUT_BF16, int N>
static hipError_t launch_dispatch_grad_t(eep_ctx* c, const void* grad_recv, void* grad_x, int T, hipStream_t st) {
  const int pieces = c->H / N, parts = (pieces + 63) / 64;
  return in_launches(T, max_blocks(64) / parts, [&](int64_t first, int64_t n) {
    hipLaunchKernelGGL((k_dispatch_grad<Y_BF16, OUT_BF16, N>), dim3((unsigned)(n * parts)), dim3(64), 0, st, c->row_of, grad_recv,
                       grad_x, c->k, pieces, (uint32_t)parts, part_magic(parts, n * parts), first);
    return hipGetLastError();
  });
}

hipError_t launch_dispatch_grad(eep_ctx* c, const void* grad_recv, void* grad_x, int T, hipStream_t st) {
  const bool yb = c->cfg.y_dtype == EEP_BF16, ob = c->cfg.out_dtype == EEP_BF16;
  if (yb && ob) return launch_dispatch_grad_t<true, true, 8>(c, grad_recv, grad_x, T, st);
  if (yb) return launch_dispatch_grad_t<true, false, 8>(c, grad_recv, grad_x, T, st);
  if (ob) return launch_dispatch_grad_t<false, true, 8>(c, grad_recv, grad_x, T, st);
  return launch_dispatch_grad_t<false, false, 4>(c, grad_recv, grad_x, T, st);
}

}  // namespace eep
