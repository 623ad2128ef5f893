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
  int* counts;                                                    // the results, or NULL (then mean and balance are too)
  float *mean, *balance;
  int* ticket;                                                    // what several blocks leave; NULL: the balance has a launch of its own
  double* loss;
  float* sums;
  int* parts;
  long long stride, rows;
  int experts, k, normalize;
};

constexpr float LOG2E = 1.44269504088896341f;

// ---- a row among L lanes ----

// Joins the values of L neighbouring lanes; all of them get the result.  Within sixteen lanes the other operand comes by the instruction's own lane exchange (DPP): neighbours,
// pairs, the mirrored eight, the mirrored sixteen.
template <int CONTROL>
__device__ __forceinline__ unsigned from_lane(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, true); }
template <int L, typename F>
__device__ __forceinline__ unsigned join(unsigned v, F&& f) {
  if constexpr (L >= 2) v = f(v, from_lane<0xB1>(v));
  if constexpr (L >= 4) v = f(v, from_lane<0x4E>(v));
  if constexpr (L >= 8) v = f(v, from_lane<0x141>(v));
  if constexpr (L >= 16) v = f(v, from_lane<0x140>(v));
  if constexpr (L >= 32) v = f(v, (unsigned)__shfl_xor((int)v, 16));
  if constexpr (L >= 64) v = f(v, (unsigned)__shfl_xor((int)v, 32));
  return v;
}
template <int L>
__device__ __forceinline__ unsigned most_of(unsigned v) { return join<L>(v, [](unsigned a, unsigned b) { return max(a, b); }); }
template <int L>
__device__ __forceinline__ unsigned least_of(unsigned v) { return join<L>(v, [](unsigned a, unsigned b) { return min(a, b); }); }
template <int L>
__device__ __forceinline__ float sum_of(float v) {
  return __uint_as_float(join<L>(__float_as_uint(v), [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// the expert of a lane's c-th logit
template <int L>
__device__ __forceinline__ int expert_of(int c) { return (c / 8 * L + (int)(threadIdx.x % L)) * 8 + c % 8; }

// Where an expert stands in a row of LDS: the halves of a lane's chunks lie apart, so that neighbouring lanes' 16 bytes are neighbours.
template <int L>
__device__ __forceinline__ int slot_of(int expert) { return expert / (8 * L) * (8 * L) + expert % 8 / 4 * (4 * L) + expert / 8 % L * 4 + expert % 4; }

// Numbers as whole numbers of the same order.  -0 counts as 0, NaN as -infinity, which keys below THERE are.  A bf16 number leaves room for its expert below it, so that keys are all
// different and equal numbers come in the experts' order.
constexpr unsigned THERE = 0x00800000u;
template <typename T>
__device__ __forceinline__ unsigned key_of(float v, int expert) {
  const int u = __float_as_int(fmaxf(v, -INFINITY) + 0.f);
  const unsigned key = (unsigned)(u ^ (u >> 31 | (int)0x80000000));
  return sizeof(T) == 4 ? key : (key & 0xffff0000u) | (0xffffu - expert);
}
template <typename T>
__device__ __forceinline__ float value_of(unsigned key) {
  const unsigned u = key >> 31 ? key & 0x7fffffffu : ~key;
  return __uint_as_float(sizeof(T) == 4 ? u : u & 0xffff0000u);
}

// A row's logits as they lie in memory, which are asked for while the row before is worked on; then as numbers (-infinity behind the row's end).
template <typename T, int L, int C>
struct Row {
  Raw8<T> raw[C / 8];
  __device__ __forceinline__ void load(const T* row, int experts) {
#pragma unroll
    for (int j = 0; j < C / 8; ++j) raw[j].template load<false>(row + expert_of<L>(j * 8), experts - expert_of<L>(j * 8));
  }
  __device__ __forceinline__ void values(int experts, float (&v)[C]) const {                       // (of rows that are not there: zeros)
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      const int left = experts - expert_of<L>(j * 8);
      float w[8];
      raw[j].values(w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j * 8 + i] = i < left ? w[i] : -INFINITY;
    }
  }
};
template <int C>
__device__ __forceinline__ unsigned most(const unsigned (&key)[C]) {
  unsigned m = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) m = max(m, key[c]);
  return m;
}
// v = exp(v - top); their sum over the row (NaN and +infinity make it NaN)
template <int L, int C>
__device__ __forceinline__ float powers(float (&v)[C], float top) {
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    v[c] = __builtin_amdgcn_exp2f((v[c] - top) * LOG2E);
    s += v[c];
  }
  return sum_of<L>(s);
}

// The row's next choice: its key (below THERE: none) and expert.  `last` is the choice before it.
template <typename T, int L, int C>
__device__ __forceinline__ unsigned next_choice(unsigned (&key)[C], unsigned last, int& expert) {
  if constexpr (sizeof(T) == 2) {
    // The largest key below the last: less the last, modulo 2^32, keys below it are above all others.
    unsigned m = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) m = max(m, key[c] - last);
    m = most_of<L>(m) + last;
    expert = m >= THERE ? (int)(0xffffu - (m & 0xffffu)) : -1;
    return m;
  } else {
    // (the key does not tell equal numbers apart: the lowest expert among them is found, and taken out)
    const unsigned m = most_of<L>(most(key));
    int mine = -1;
#pragma unroll
    for (int c = C - 1; c >= 0; --c) mine = key[c] == m ? c : mine;
    const unsigned at = mine >= 0 ? (unsigned)((mine / 8 * L + (int)(threadIdx.x % L)) * 8 + mine % 8) : 0xffffffffu, first = least_of<L>(at);
    mine = at == first ? mine : -1;
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] = c == mine ? 0u : key[c];
    expert = m >= THERE ? (int)first : -1;
    return m;
  }
}

// ---- counts, means, balance ----

constexpr int SUM_EXPERTS = 8;                                    // of a block of route_sum_kernel

template <typename T, int L, int C, bool STATS>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a) {
  constexpr int R = 256 / L;                                      // rows of a block at a time
  extern __shared__ __align__(16) unsigned char lds[];
  int* ids = (int*)lds;                                           // (where a row has fewer lanes than it may have choices)
  float* weights = (float*)lds + (L < MOST_CHOICES ? R * a.k : 0);
  int* hist = (int*)(weights + (L < MOST_CHOICES ? R * a.k : 0));
  float* wide = (float*)hist + (a.experts + 1);
  float total[C];
  if constexpr (STATS) {
#pragma unroll
    for (int c = 0; c < C; ++c) total[c] = 0.f;
    for (int e = threadIdx.x; e <= a.experts; e += 256) hist[e] = 0;
    __syncthreads();
  }
  const int at = threadIdx.x / L, lane = threadIdx.x % L;
  Row<T, L, C> next;
  const auto ask = [&](long long row) { next.load((const T*)a.logits + (row < a.rows ? row : 0) * a.stride, row < a.rows ? a.experts : 0); };
  ask((long long)blockIdx.x * R + at);
  for (long long first = (long long)blockIdx.x * R; first < a.rows; first += (long long)gridDim.x * R) {
    const long long row = first + at;
    const bool in = row < a.rows;
    float v[C];
    unsigned key[C];
    next.values(a.experts, v);
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] = key_of<T>(v[c], expert_of<L>(c));
    ask(row + (long long)gridDim.x * R);
    const unsigned best = in ? most_of<L>(most(key)) : 0u;
    const float top = value_of<T>(best), inv = 1.f / powers<L>(v, top);
    if constexpr (STATS) {
      if (best >= THERE) {
#pragma unroll
        for (int c = 0; c < C; ++c) total[c] += v[c] * inv;
        if (lane == 0) atomicAdd(&hist[a.experts], 1);
      }
    }
    // (where a row has as many lanes as it may have choices, lane j has the j-th: its key and expert)
    float of_all = 0.f;
    int my_id = -1;
    unsigned m = best, my_key = 0;
    for (int j = 0; j < a.k; ++j) {
      int id = -1;
      if (m >= THERE) {                                           // (behind the last expert that is there all are none)
        if (j == 0 && sizeof(T) == 2) id = (int)(0xffffu - (m & 0xffffu));
        else m = next_choice<T, L, C>(key, m, id);
      }
      if constexpr (L >= MOST_CHOICES) {
        my_id = lane == j ? id : my_id;
        my_key = lane == j ? m : my_key;
      } else {
        const float p = m >= THERE ? __builtin_amdgcn_exp2f((value_of<T>(m) - top) * LOG2E) * inv : 0.f;
        of_all += p;
        if (lane == 0) {
          ids[at * a.k + j] = id;
          weights[at * a.k + j] = p;
          if (STATS && id >= 0) atomicAdd(&hist[id], 1);
        }
      }
    }
    if constexpr (L >= MOST_CHOICES) {
      const float p = my_id >= 0 ? __builtin_amdgcn_exp2f((value_of<T>(my_key) - top) * LOG2E) * inv : 0.f;
      if (a.normalize) of_all = sum_of<L>(p);
      if (in && lane < a.k) {
        if (STATS && my_id >= 0) atomicAdd(&hist[my_id], 1);
        a.expert[row * a.k + lane] = my_id;
        if (a.weight) a.weight[row * a.k + lane] = a.normalize && my_id >= 0 ? p / of_all : p;
      }
    } else {
      if (a.normalize && lane == 0 && best >= THERE)
        for (int j = 0; j < a.k && ids[at * a.k + j] >= 0; ++j) weights[at * a.k + j] /= of_all;  // (0 behind them, also where of_all is NaN)
      __syncthreads();
      const int n = (int)(a.rows - first < R ? a.rows - first : R) * a.k;
      for (int i = threadIdx.x; i < n; i += 256) {
        a.expert[first * a.k + i] = ids[i];
        if (a.weight) a.weight[first * a.k + i] = weights[i];
      }
      __syncthreads();
    }
  }
  if constexpr (STATS) {
    // the rows of a wave first, then the four waves in order
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int d = L; d < 64; d *= 2) total[c] += __shfl_xor(total[c], d);
    __syncthreads();
    for (int w = 0; w < 4; ++w) {
      if ((int)(threadIdx.x >> 6) == w && (threadIdx.x & 63) < L)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int e = expert_of<L>(c);
          if (e < a.experts) wide[e] = w ? wide[e] + total[c] : total[c];
        }
      __syncthreads();
    }
    if (gridDim.x > 1) {
      if (a.ticket && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
      for (int e = threadIdx.x; e < a.experts; e += 256) a.sums[(long long)blockIdx.x * a.experts + e] = wide[e];
      for (int e = threadIdx.x; e <= a.experts; e += 256) a.parts[(long long)blockIdx.x * (a.experts + 1) + e] = hist[e];
      return;
    }
    // the only block
    __shared__ double loss[4];
    __shared__ int all[4];
    const int counted = hist[a.experts];
    double mine = 0;
    int chosen = 0;
    for (int e = threadIdx.x; e <= a.experts; e += 256) {
      a.counts[e] = hist[e];
      if (e == a.experts) break;
      const double p = (double)wide[e] / (counted > 0 ? counted : 1);
      if (a.mean) a.mean[e] = (float)p;
      mine += hist[e] * p;
      chosen += hist[e];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      mine += __shfl_xor(mine, d);
      chosen += __shfl_xor(chosen, d);
    }
    if ((threadIdx.x & 63) == 0) {
      loss[threadIdx.x >> 6] = mine;
      all[threadIdx.x >> 6] = chosen;
    }
    __syncthreads();
    if (threadIdx.x == 0 && a.balance) {
      const long long n = (long long)all[0] + all[1] + all[2] + all[3];
      *a.balance = (float)(n > 0 ? (loss[0] + loss[1] + loss[2] + loss[3]) * a.experts / (double)n : 0.0);
    }
  }
}

// Counts, means and the balance loss from the blocks' sums: a block for eight experts (128 threads each, a load of up to 1024 blocks' sums at a time).  Their shares of the loss are added up in
// order by the last block to come, whose order of memory costs a write-back of the caches, or (no ticket) by a launch of its own: 65536 rows, 256 experts 12.4 us, 7.2 + 4 in two launches, a pass
// 60, 57; 6397 rows of 100: 7.0, 4.9 + 1.4, but a pass, whose time is the host's, 25.5, 28.5.  (Blocks of 32 experts: 16.2.)
__global__ __launch_bounds__(1024) void route_sum_kernel(RouteArgs a, int blocks) {
  __shared__ int n[16][SUM_EXPERTS], rows[16];
  __shared__ double d[16][SUM_EXPERTS];
  const int c = threadIdx.x % SUM_EXPERTS, s = threadIdx.x / SUM_EXPERTS, wave = threadIdx.x >> 6, l = threadIdx.x & 63, e = blockIdx.x * SUM_EXPERTS + c;
  constexpr int SLICES = 1024 / SUM_EXPERTS;
  int counted = 0, t = 0;
  double p = 0;
  for (int b = threadIdx.x; b < blocks; b += 1024) counted += a.parts[(long long)b * (a.experts + 1) + a.experts];
  if (e < a.experts)
    for (int b = s; b < blocks; b += SLICES * 8) {
      int m[8];
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = b + SLICES * i < blocks;
        m[i] = in ? a.parts[(long long)(b + SLICES * i) * (a.experts + 1) + e] : 0;
        f[i] = in ? a.sums[(long long)(b + SLICES * i) * a.experts + e] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) t += m[i], p += f[i];
    }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    counted += __shfl_xor(counted, x);
    if (x >= SUM_EXPERTS) {
      t += __shfl_xor(t, x);
      p += __shfl_xor(p, x);
    }
  }
  if (l < SUM_EXPERTS) n[wave][l] = t, d[wave][l] = p;
  if (l == 0) rows[wave] = counted;
  __syncthreads();
  if (threadIdx.x >= SUM_EXPERTS) return;
  counted = rows[0];
#pragma unroll
  for (int w = 1; w < 16; ++w) t += n[w][c], p += d[w][c], counted += rows[w];
  p /= counted > 0 ? counted : 1;
  if (e < a.experts) {
    a.counts[e] = t;
    if (a.mean) a.mean[e] = (float)p;
  }
  double share = t * p, all = t;
#pragma unroll
  for (int x = 1; x < SUM_EXPERTS; x *= 2) {
    share += __shfl_xor(share, x);
    all += __shfl_xor(all, x);
  }
  if (threadIdx.x > 0) return;
  if (blockIdx.x == 0) a.counts[a.experts] = counted;
  if (!a.ticket) {
    a.loss[2 * blockIdx.x] = share;
    a.loss[2 * blockIdx.x + 1] = all;
    return;
  }
  __hip_atomic_store(&a.loss[2 * blockIdx.x], share, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(&a.loss[2 * blockIdx.x + 1], all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (__hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) != (int)gridDim.x - 1 || !a.balance) return;
  share = all = 0;
  for (int b = 0; b < (int)gridDim.x; ++b) {
    share += __hip_atomic_load(&a.loss[2 * b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all += __hip_atomic_load(&a.loss[2 * b + 1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  *a.balance = (float)(all > 0 ? share * a.experts / all : 0);
}

__global__ __launch_bounds__(64) void route_balance_kernel(const double* loss, int blocks, int experts, float* balance) {
  double share = 0, all = 0;
  for (int b = threadIdx.x; b < blocks; b += 64) share += loss[2 * b], all += loss[2 * b + 1];
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    share += __shfl_xor(share, x);
    all += __shfl_xor(all, x);
  }
  if (threadIdx.x == 0) *balance = (float)(all > 0 ? share * experts / all : 0);
}

// without rows
__global__ void route_none_kernel(int experts, int* counts, float* mean, float* balance) {
  for (int e = threadIdx.x; e <= experts; e += 256) {
    counts[e] = 0;
    if (mean && e < experts) mean[e] = 0.f;
  }
  if (balance && threadIdx.x == 0) *balance = 0.f;
}

// ---- gradient ----

struct RouteBackArgs {
  const void* logits;
  const int *expert, *counts;
  const float* dweight;
  void* dlogits;
  long long stride, dstride, rows;
  int experts, k, normalize;
  float balance_grad;
};

// dl_e = p_e (share_e - D) + extra_e, share_e = c counts_e.  extra is zero but for the choices, which are a lane's each: p_e g_e (then their sum is in D), or that of the softmax over
// the choices, w_e (g_e - sum_j w_j g_j) with w_e = p_e / the choices' p.  The choices' p come from the lanes that hold their logits through a row of LDS, and extra goes back through another
// (65536 rows, 256 experts, 8 choices in bf16: 25 us; with compares of every logit with every choice 97, with the choices' logits read again from memory 29).
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void route_back_kernel(RouteBackArgs a) {
  constexpr int R = 256 / L, EACH = L < MOST_CHOICES ? MOST_CHOICES / L : 1;      // choices of a lane
  constexpr bool P_ROWS = R * L * C * 4 <= 32768;                 // (the p of longer rows' choices are formed again)
  __shared__ __align__(16) float rows_extra[R][L * C], rows_p[P_ROWS ? R : 1][P_ROWS ? L * C : 1];
  __shared__ int part[4];
  const int at = threadIdx.x / L, lane = threadIdx.x % L;
  float *extra = rows_extra[at], *ps = rows_p[P_ROWS ? at : 0];
#pragma unroll
  for (int c = 0; c < C; ++c) extra[slot_of<L>(expert_of<L>(c))] = 0.f;
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
  __syncthreads();
  const auto settle = [] {                                        // (what lanes of a wave wrote to LDS is there for the others)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  Row<T, L, C> next;
  int next_id[EACH];
  float next_g[EACH];
  const auto ask = [&](long long row) {
    const bool in = row < a.rows;
    next.load((const T*)a.logits + (in ? row : 0) * a.stride, in ? a.experts : 0);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = lane + i * L;
      const bool is = a.dweight && in && j < a.k;
      next_id[i] = is ? a.expert[row * a.k + j] : -1;
      next_g[i] = is ? a.dweight[row * a.k + j] : 0.f;
    }
  };
  ask((long long)blockIdx.x * R + at);
  for (long long first = (long long)blockIdx.x * R; first < a.rows; first += (long long)gridDim.x * R) {
    const long long row = first + at;
    const bool in = row < a.rows;
    int id[EACH];
    float g[EACH], l[EACH], v[C];
    next.values(a.experts, v);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      id[i] = (unsigned)next_id[i] < (unsigned)a.experts ? next_id[i] : -1;
      g[i] = next_g[i];
    }
    ask(row + (long long)gridDim.x * R);
    // (what is NaN or -infinity is not there; the largest of the others)
    unsigned there[(C + 31) / 32] = {};
    float top = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      there[c / 32] |= (v[c] > -INFINITY ? 1u : 0u) << c % 32;
      top = fmaxf(top, v[c]);
    }
    top = __uint_as_float(join<L>(__float_as_uint(top), [](unsigned a, unsigned b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
    const float inv = 1.f / powers<L>(v, top);
    float mean = 0.f, of_chosen = 0.f, of_weights = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      v[c] *= inv;                                                // (0 where there is none, unless the row is left out or NaN)
      mean += v[c] * share[c];
    }
    if constexpr (P_ROWS) {
#pragma unroll
      for (int c = 0; c < C; c += 4) *reinterpret_cast<float4*>(ps + slot_of<L>(expert_of<L>(c))) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
      settle();
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if constexpr (P_ROWS) {
        l[i] = id[i] >= 0 ? ps[slot_of<L>(id[i])] : 0.f;
      } else {
        const float logit = id[i] >= 0 ? to_float(((const T*)a.logits)[row * a.stride + id[i]]) : 0.f;
        l[i] = id[i] >= 0 && logit > -INFINITY ? __builtin_amdgcn_exp2f((logit - top) * LOG2E) * inv : 0.f;
      }
      of_chosen += l[i];
      of_weights += id[i] >= 0 ? l[i] * g[i] : 0.f;
    }
    mean = sum_of<L>(mean);
    of_weights = sum_of<L>(of_weights);
    if (a.normalize) {
      const float over = 1.f / sum_of<L>(of_chosen);
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (id[i] >= 0) extra[slot_of<L>(id[i])] = l[i] * over * (g[i] - of_weights * over);
    } else {
      mean += of_weights;
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (id[i] >= 0) extra[slot_of<L>(id[i])] = l[i] * g[i];
    }
    settle();
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      const int e = expert_of<L>(j * 8);
      float d[8];
      const float4 x = *reinterpret_cast<const float4*>(extra + slot_of<L>(e)), y = *reinterpret_cast<const float4*>(extra + slot_of<L>(e + 4));
      const float more[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = j * 8 + i;
        d[i] = there[c / 32] >> c % 32 & 1 ? v[c] * (share[c] - mean) + more[i] : 0.f;
      }
      store8<T, false>((T*)a.dlogits + (in ? row : 0) * a.dstride + e, in ? a.experts - e : 0, d);
    }
    settle();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (id[i] >= 0) extra[slot_of<L>(id[i])] = 0.f;
  }
}

// Lanes of a row and logits of a lane.
template <typename F>
void with_lanes(int experts, F&& go) {
  typedef std::integral_constant<int, 8> Eight;
  if (experts <= 8) go(std::integral_constant<int, 1>(), Eight());
  else if (experts <= 32) go(std::integral_constant<int, 4>(), Eight());
  else if (experts <= 128) go(std::integral_constant<int, 16>(), Eight());
  else if (experts <= 256) go(std::integral_constant<int, 16>(), std::integral_constant<int, 16>());
  else if (experts <= 512) go(std::integral_constant<int, 16>(), std::integral_constant<int, 32>());
  else if (experts <= 1024) go(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
  else go(std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
}
long long tiles_of(long long rows, int experts) {
  const int r = 256 / (experts <= 8 ? 1 : experts <= 32 ? 4 : experts <= 512 ? 16 : 64);
  return (rows + r - 1) / r;
}
constexpr int LOSS_AT = 16, SUMS_AT = LOSS_AT + MOST_EXPERTS / SUM_EXPERTS * 16;       // in the workspace, behind the ticket
// As many blocks as are on the chip together: each has what it leaves behind, or the counts, to see to once (65536 rows of 64 experts, gradient: 13.8 us with 1024 blocks, 17.1 with 512; 16384 of
// 512: 20.2 with 512, 27.7 with 1024, and forward with counts 26.5, 37).
int most_blocks(long long rows, int experts) { return (int)std::min(tiles_of(rows, experts), experts > 1024 ? 256ll : experts > 256 && experts <= 512 ? 512ll : 1024ll); }

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
  const int blocks = most_blocks(rows, experts);
  return blocks > 1 ? SUMS_AT + (int64_t)blocks * (2 * experts + 1) * 4 : 0;
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
  if (rows == 0) {
    hipLaunchKernelGGL(route_none_kernel, dim3(1), dim3(256), 0, st, experts, counts, mean, balance);
    return operator_launched();
  }
  const int blocks = most_blocks(rows, experts);
  const bool apart = (long long)blocks * experts >= 1 << 17;
  uint8_t* const w = (uint8_t*)work;
  float* const sums = (float*)(w + SUMS_AT);
  const RouteArgs a = {logits, expert, weight, counts, mean, balance, apart ? nullptr : (int*)w, (double*)(w + LOSS_AT), sums, (int*)(sums + (long long)blocks * experts), logits_stride, rows, experts, k, normalize};
  with_lanes(experts, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value;
    const unsigned lds = ((L < MOST_CHOICES ? 2 * (256 / L) * k : 0) + (counts ? 2 * experts + 1 : 0)) * 4;
    const dim3 grid(counts ? (unsigned)blocks : (unsigned)std::min(tiles_of(rows, experts), 1ll << 20));
    const auto go = [&](auto t) {
      typedef decltype(t) T;
      if (counts) hipLaunchKernelGGL((route_kernel<T, L, C, true>), grid, dim3(256), lds, st, a);
      else hipLaunchKernelGGL((route_kernel<T, L, C, false>), grid, dim3(256), lds, st, a);
    };
    if (precision == GAN_FP32) go(float());
    else go(bf16_t());
  });
  if (counts && blocks > 1) {
    const int sum_blocks = (experts + SUM_EXPERTS - 1) / SUM_EXPERTS;
    hipLaunchKernelGGL(route_sum_kernel, dim3(sum_blocks), dim3(1024), 0, st, a, blocks);
    if (balance && apart) hipLaunchKernelGGL(route_balance_kernel, dim3(1), dim3(64), 0, st, (const double*)(w + LOSS_AT), sum_blocks, experts, balance);
  }
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
    const dim3 grid((unsigned)most_blocks(rows, experts));
    if (precision == GAN_FP32) hipLaunchKernelGGL((route_back_kernel<float, L, C>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((route_back_kernel<bf16_t, L, C>), grid, dim3(256), 0, st, a);
  });
  return operator_launched();
}
