// The router: a row's k best experts, their weights, how many rows every expert gets, and the balance loss; and the gradient.
//
//   p_e = exp(l_e - max) / sum over the experts that are there of the same;   there: l_e > -infinity (and no NaN)
//   weight of a choice: its p, or (normalize) its p over those of all choices
//   balance = experts * sum_e counts_e / sum(counts) * mean_e,   mean_e = the mean of p_e over the rows that have an expert at all
//
// Gradient, with g_e the weight's gradient where e is chosen and c = balance_grad * experts / sum(counts) / rows counted:
//   dl_e = p_e (d_e - sum_j p_j d_j),   d_e = c counts_e + g_e                           (normalize: g through the softmax over the choices instead)
//
// Bound by the instructions of the selection (k rounds of a maximum over the row) where k is large, else by memory: one pass over the logits.  L lanes hold a row, eight neighbouring logits a
// chunk; rows stand side by side in a wave, so that narrow rows leave no lanes idle.
#include "operators.h"

#include <algorithm>
#include <type_traits>

namespace gan {
namespace {

constexpr int MOST_CHOICES = 16, MOST_EXPERTS = 4096;

struct RouteArgs {
  const void* logits;
  int* expert;
  float* weight;
  float* sums;                                                    // [blocks][experts]: of the probabilities, or NULL
  int* counts;                                                    // [blocks][experts + 1]: choices of each expert, and rows that have one
  long long stride, rows;
  int experts, k, normalize;
};

// Numbers as whole numbers of the same order; 0: not there.  -0 counts as 0.
__device__ __forceinline__ unsigned key_of(float v) {
  const unsigned u = __float_as_uint(v + 0.f);
  return v > -INFINITY ? (u >> 31 ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }

template <int L>
__device__ __forceinline__ unsigned most_of(unsigned v) {
#pragma unroll
  for (int d = 1; d < L; d *= 2) v = max(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}
template <int L>
__device__ __forceinline__ unsigned least_of(unsigned v) {
#pragma unroll
  for (int d = 1; d < L; d *= 2) v = min(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}
template <int L>
__device__ __forceinline__ float sum_of(float v) {
#pragma unroll
  for (int d = 1; d < L; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// the expert of a lane's c-th logit
template <int L>
__device__ __forceinline__ int expert_of(int c) { return (c / 8 * L + (int)(threadIdx.x % L)) * 8 + c % 8; }

// A row's keys; true where one of its logits is NaN.
template <typename T, int L, int C>
__device__ __forceinline__ bool load_keys(const T* row, int experts, bool in, unsigned (&key)[C]) {
  bool bad = false;
#pragma unroll
  for (int j = 0; j < C / 8; ++j) {
    const int e = expert_of<L>(j * 8);
    float v[8];
    load8<T, false>(row + e, in ? experts - e : 0, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool is = in && e + i < experts;
      key[j * 8 + i] = is ? key_of(v[i]) : 0u;
      bad |= is && v[i] != v[i];
    }
  }
  return bad;
}

template <typename T, int L, int C, bool STATS>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a) {
  constexpr int R = 256 / L;                                      // rows of a block at a time
  extern __shared__ __align__(16) unsigned char lds[];
  int* ids = (int*)lds;
  float* weights = (float*)lds + R * a.k;
  int* hist = (int*)lds + 2 * R * a.k;
  float* wide = (float*)hist + (a.experts + 1);
  float total[C];
  if constexpr (STATS) {
#pragma unroll
    for (int c = 0; c < C; ++c) total[c] = 0.f;
    for (int e = threadIdx.x; e <= a.experts; e += 256) hist[e] = 0;
    __syncthreads();
  }
  const int at = threadIdx.x / L, lane = threadIdx.x % L;
  for (long long first = (long long)blockIdx.x * R; first < a.rows; first += (long long)gridDim.x * R) {
    const long long row = first + at;
    const bool in = row < a.rows;
    unsigned key[C];
    const bool bad = load_keys<T, L, C>((const T*)a.logits + (in ? row : 0) * a.stride, a.experts, in, key);
    unsigned best = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) best = max(best, key[c]);
    best = most_of<L>(best);
    const float top = value_of(best);
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) s += key[c] ? expf(value_of(key[c]) - top) : 0.f;
    s = sum_of<L>(s);
    if (most_of<L>(bad)) s = NAN;
    const float inv = 1.f / s;
    if constexpr (STATS) {
      if (best) {
#pragma unroll
        for (int c = 0; c < C; ++c) total[c] += key[c] ? expf(value_of(key[c]) - top) * inv : 0.f;
        if (lane == 0) atomicAdd(&hist[a.experts], 1);
      }
    }
    float of_all = 0.f;
    for (int j = 0; j < a.k; ++j) {
      unsigned m = 0, index = 0xffffffffu;
#pragma unroll
      for (int c = 0; c < C; ++c) m = max(m, key[c]);
      m = most_of<L>(m);
#pragma unroll
      for (int c = 0; c < C; ++c) index = min(index, key[c] == m ? (unsigned)expert_of<L>(c) : 0xffffffffu);
      index = least_of<L>(index);
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] = (unsigned)expert_of<L>(c) == index ? 0u : key[c];
      const float p = m ? expf(value_of(m) - top) * inv : 0.f;
      of_all += p;
      if (lane == 0) {
        ids[at * a.k + j] = m ? (int)index : -1;
        weights[at * a.k + j] = p;
        if (STATS && m) atomicAdd(&hist[index], 1);
      }
    }
    if (a.normalize && lane == 0 && best)
      for (int j = 0; j < a.k; ++j) weights[at * a.k + j] /= of_all;
    __syncthreads();
    const int n = (int)(a.rows - first < R ? a.rows - first : R) * a.k;
    for (int i = threadIdx.x; i < n; i += 256) {
      a.expert[first * a.k + i] = ids[i];
      if (a.weight) a.weight[first * a.k + i] = weights[i];
    }
    __syncthreads();
  }
  if constexpr (STATS) {
    // the rows of a wave first, then the four waves in order
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int d = L; d < 64; d *= 2) total[c] += __shfl_xor(total[c], d);
    for (int w = 0; w < 4; ++w) {
      if ((int)(threadIdx.x >> 6) == w && (threadIdx.x & 63) < L)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int e = expert_of<L>(c);
          if (e < a.experts) wide[e] = w ? wide[e] + total[c] : total[c];
        }
      __syncthreads();
    }
    for (int e = threadIdx.x; e < a.experts; e += 256) a.sums[(long long)blockIdx.x * a.experts + e] = wide[e];
    for (int e = threadIdx.x; e <= a.experts; e += 256) a.counts[(long long)blockIdx.x * (a.experts + 1) + e] = hist[e];
  }
}

// counts, means and the balance loss from the blocks' sums
__global__ __launch_bounds__(1024) void route_sum_kernel(const float* sums, const int* parts, int blocks, int experts, int* counts, float* mean, float* balance) {
  __shared__ int n[32][33];
  __shared__ double d[32][33];
  __shared__ int rows;
  const int c = threadIdx.x & 31, s = threadIdx.x >> 5;
  int counted = 0;
  for (int b = threadIdx.x; b < blocks; b += 1024) counted += parts[(long long)b * (experts + 1) + experts];
  n[s][c] = counted;
  __syncthreads();
  if (threadIdx.x == 0) {
    int t = 0;
    for (int i = 0; i < 1024; ++i) t += n[i >> 5][i & 31];
    rows = t;
    counts[experts] = t;
  }
  __syncthreads();
  double loss = 0;
  long long all = 0;
  for (int e0 = 0; e0 < experts; e0 += 32) {
    const int e = e0 + c;
    int t = 0;
    double p = 0;
    if (e < experts)
      for (int b = s; b < blocks; b += 32) {
        t += parts[(long long)b * (experts + 1) + e];
        p += sums[(long long)b * experts + e];
      }
    __syncthreads();
    n[s][c] = t;
    d[s][c] = p;
    __syncthreads();
    if (s == 0 && e < experts) {
      for (int i = 1; i < 32; ++i) t += n[i][c], p += d[i][c];
      p /= rows > 0 ? rows : 1;
      counts[e] = t;
      if (mean) mean[e] = (float)p;
      loss += t * p;
      all += t;
    }
  }
  __syncthreads();
  if (s == 0) {
    d[0][c] = loss;
    d[1][c] = (double)all;
  }
  __syncthreads();
  if (threadIdx.x == 0 && balance) {
    for (int i = 1; i < 32; ++i) loss += d[0][i], all += (long long)d[1][i];
    *balance = (float)(all > 0 ? loss * experts / (double)all : 0);
  }
}

struct RouteBackArgs {
  const void* logits;
  const int *expert, *counts;
  const float* dweight;
  void* dlogits;
  long long stride, dstride, rows;
  int experts, k, normalize;
  float balance_grad;
};

template <typename T, int L, int C>
__global__ __launch_bounds__(256) void route_back_kernel(RouteBackArgs a) {
  constexpr int R = 256 / L;
  __shared__ int part[4];
  float share[C];
#pragma unroll
  for (int c = 0; c < C; ++c) share[c] = 0.f;
  if (a.counts) {
    int all = 0;
    for (int e = threadIdx.x; e < a.experts; e += 256) all += a.counts[e];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = all;
    __syncthreads();
    all = part[0] + part[1] + part[2] + part[3];
    const int counted = a.counts[a.experts];
    const float coefficient = all > 0 && counted > 0 ? a.balance_grad * (float)a.experts / (float)all / (float)counted : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = expert_of<L>(c);
      share[c] = e < a.experts ? coefficient * (float)a.counts[e] : 0.f;
    }
  }
  const int at = threadIdx.x / L;
  for (long long first = (long long)blockIdx.x * R; first < a.rows; first += (long long)gridDim.x * R) {
    const long long row = first + at;
    const bool in = row < a.rows;
    unsigned key[C];
    const bool bad = load_keys<T, L, C>((const T*)a.logits + (in ? row : 0) * a.stride, a.experts, in, key);
    float g[C], p[C];
    unsigned chosen[(C + 31) / 32] = {};
#pragma unroll
    for (int c = 0; c < C; ++c) g[c] = 0.f;
    if (a.dweight && in)
      for (int j = 0; j < a.k; ++j) {
        const int e = a.expert[row * a.k + j];
        const float dw = a.dweight[row * a.k + j];
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (expert_of<L>(c) == e) {
            g[c] += dw;
            chosen[c / 32] |= 1u << c % 32;
          }
      }
    unsigned best = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) best = max(best, key[c]);
    best = most_of<L>(best);
    const float top = value_of(best);
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      p[c] = key[c] ? expf(value_of(key[c]) - top) : 0.f;
      s += p[c];
    }
    s = sum_of<L>(s);
    if (most_of<L>(bad)) s = NAN;
    const float inv = 1.f / s;
    float mean = 0.f, of_chosen = 0.f, of_weights = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      p[c] = key[c] ? p[c] * inv : 0.f;
      const bool is = chosen[c / 32] >> c % 32 & 1;
      if (a.normalize) {
        of_chosen += is ? p[c] : 0.f;
        of_weights += is ? p[c] * g[c] : 0.f;
        mean += p[c] * share[c];
      } else {
        mean += p[c] * (share[c] + g[c]);
      }
    }
    mean = sum_of<L>(mean);
    float over = 0.f, mean_weights = 0.f;
    if (a.normalize) {
      of_chosen = sum_of<L>(of_chosen);
      of_weights = sum_of<L>(of_weights);
      over = 1.f / of_chosen;
      mean_weights = of_weights * over;
    }
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = j * 8 + i;
        const bool is = chosen[c / 32] >> c % 32 & 1;
        if (a.normalize) d[i] = p[c] * (share[c] - mean) + (is && key[c] ? p[c] * over * (g[c] - mean_weights) : 0.f);
        else d[i] = p[c] * (share[c] + g[c] - mean);
        if (!key[c]) d[i] = 0.f;
      }
      const int e = expert_of<L>(j * 8);
      store8<T, false>((T*)a.dlogits + (in ? row : 0) * a.dstride + e, in ? a.experts - e : 0, d);
    }
  }
}

// lanes of a row
int lanes_of(int experts) { return experts <= 8 ? 1 : experts <= 32 ? 4 : experts <= 128 ? 16 : 64; }
long long tiles_of(long long rows, int experts) {
  const int r = 256 / lanes_of(experts);
  return (rows + r - 1) / r;
}
// Blocks that leave sums of their rows behind.
int stat_blocks(long long rows, int experts) { return (int)std::min(tiles_of(rows, experts), 512ll); }

template <typename F>
void with_lanes(int experts, F&& go) {
  if (experts <= 8) go(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
  else if (experts <= 32) go(std::integral_constant<int, 4>(), std::integral_constant<int, 8>());
  else if (experts <= 128) go(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
  else if (experts <= 512) go(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
  else if (experts <= 1024) go(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
  else go(std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
}

gan_status check_route(int32_t precision, int64_t rows, int32_t experts, int32_t k, int64_t stride) {
  if (const gan_status s = check_sizes(precision, rows, experts)) return s;
  if (k < 1 || k > experts) return operator_fail(GAN_E_ARG, "k is below one or above the number of experts");
  if (stride < experts) return operator_fail(GAN_E_ARG, "a row's stride is below the number of experts");
  if (experts > MOST_EXPERTS || k > MOST_CHOICES) return operator_fail(GAN_E_SHAPE, "more than 4096 experts or 16 choices");
  if (rows * k > MOST_ROWS) return operator_fail(GAN_E_SHAPE, "more than 2^30 choices");
  return GAN_OK;
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" int64_t gan_route_bytes(int64_t rows, int32_t experts) {
  if (rows < 1 || experts < 1 || rows > MOST_ROWS || experts > MOST_EXPERTS) return 0;
  return (int64_t)stat_blocks(rows, experts) * (2 * experts + 1) * 4;
}

extern "C" gan_status gan_route(int32_t precision, const void* logits, int64_t logits_stride, int64_t rows, int32_t experts, int32_t k, int32_t normalize, int32_t* expert,
                                float* weight, int32_t* counts, float* mean, float* balance, void* work, int64_t work_bytes, void* hip_stream) {
  if (const gan_status s = check_route(precision, rows, experts, k, logits_stride)) return s;
  if (rows > 0 && (!logits || !expert)) return operator_fail(GAN_E_ARG, "logits or expert is NULL");
  if ((mean || balance) && !counts) return operator_fail(GAN_E_ARG, "mean and balance go with counts, which is NULL");
  const int64_t need = gan_route_bytes(rows, experts);
  if (counts && (work_bytes < need || (need > 0 && !work) || !aligned16(work))) return operator_fail(GAN_E_ARG, "work is smaller than gan_route_bytes, or not 16-byte aligned");
  if (rows == 0 && !counts) return GAN_OK;
  operator_launches();
  const hipStream_t st = (hipStream_t)hip_stream;
  const int blocks = rows > 0 ? stat_blocks(rows, experts) : 0;
  float* sums = (float*)work;
  int* parts = (int*)work + (long long)blocks * experts;
  if (rows > 0) {
    const RouteArgs a = {logits, expert, weight, sums, parts, logits_stride, rows, experts, k, normalize};
    with_lanes(experts, [&](auto l, auto c) {
      constexpr int L = decltype(l)::value, C = decltype(c)::value;
      const unsigned lds = (2 * (256 / L) * k + (counts ? 2 * experts + 1 : 0)) * 4;
      const dim3 grid(counts ? (unsigned)blocks : (unsigned)std::min(tiles_of(rows, experts), 1ll << 20));
      const auto go = [&](auto t) {
        typedef decltype(t) T;
        if (counts) hipLaunchKernelGGL((route_kernel<T, L, C, true>), grid, dim3(256), lds, st, a);
        else hipLaunchKernelGGL((route_kernel<T, L, C, false>), grid, dim3(256), lds, st, a);
      };
      if (precision == GAN_FP32) go(float());
      else go(bf16_t());
    });
  }
  if (counts) hipLaunchKernelGGL(route_sum_kernel, dim3(1), dim3(1024), 0, st, sums, parts, blocks, experts, counts, mean, balance);
  return operator_launched();
}

extern "C" gan_status gan_route_backward(int32_t precision, const void* logits, int64_t logits_stride, int64_t rows, int32_t experts, int32_t k, int32_t normalize,
                                         const int32_t* expert, const float* dweight, const int32_t* counts, float balance_grad, void* dlogits, int64_t dlogits_stride,
                                         void* hip_stream) {
  if (const gan_status s = check_route(precision, rows, experts, k, std::min(logits_stride, dlogits_stride))) return s;
  if (rows > 0 && (!logits || !dlogits || (dweight && !expert))) return operator_fail(GAN_E_ARG, "logits, dlogits or expert is NULL");
  if (rows == 0) return GAN_OK;
  operator_launches();
  const RouteBackArgs a = {logits, expert, counts, dweight, dlogits, logits_stride, dlogits_stride, rows, experts, k, normalize, balance_grad};
  const hipStream_t st = (hipStream_t)hip_stream;
  with_lanes(experts, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value;
    const dim3 grid((unsigned)std::min(tiles_of(rows, experts), 4096ll));
    if (precision == GAN_FP32) hipLaunchKernelGGL((route_back_kernel<float, L, C>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((route_back_kernel<bf16_t, L, C>), grid, dim3(256), 0, st, a);
  });
  return operator_launched();
}
