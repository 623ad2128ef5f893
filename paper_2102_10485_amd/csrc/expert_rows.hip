// Rows sorted by label on the device, handed out to their experts and put together again.
//
//   order[place[i]] = i, the labels of order[0], order[1], ... do not decrease, equal ones keep their order;   offs[g] = how many labels are below g
//   hand out      out[place[i][s]] = x[i]
//   put together  y[i] = residual[i] + sum_s weight[i][s] out[place[i][s]]
//   its gradient  dout[place[i][s]] = weight[i][s] dy[i],   dweight[i][s] = dy[i] . out[place[i][s]];     that of handing out is putting together without weights
//
// The sort is a counting sort: blocks count the labels of their stretch, a wave per label adds up the blocks before each, and the blocks place their labels.  The rest is bound by memory: every
// row is read and written once, whole rows at a time wherever they lie.
#include "group_tiles.h"
#include "row_chunks.h"

#include <algorithm>

namespace gan {
namespace {

constexpr int MOST_LABELS = 4096;
constexpr int STRETCH = 2048;                                     // labels of a block

struct SortArgs {
  const int* labels;
  int *offs, *order, *place;
  int* before;                                                    // [groups + 1][blocks]: counts; with more blocks than FUSED, the sums of the blocks before
  int* all;                                                       // [groups + 1]
  int n, groups, blocks, bits;                                    // bits: of groups
};

__device__ __forceinline__ int label_of(const SortArgs& a, int i) {
  const int g = a.labels[i];
  return (unsigned)g < (unsigned)a.groups ? g : a.groups;
}

__global__ __launch_bounds__(1024) void sort_count_kernel(SortArgs a) {
  extern __shared__ int count[];
  for (int g = threadIdx.x; g <= a.groups; g += 1024) count[g] = 0;
  __syncthreads();
  const int begin = blockIdx.x * STRETCH, end = min(a.n, begin + STRETCH);
  for (int i = begin + threadIdx.x; i < end; i += 1024) atomicAdd(&count[label_of(a, i)], 1);
  __syncthreads();
  for (int g = threadIdx.x; g <= a.groups; g += 1024) a.before[(long long)g * a.blocks + blockIdx.x] = count[g];
}

__global__ __launch_bounds__(256) void sort_scan_kernel(SortArgs a) {
  const int g = blockIdx.x * 4 + (threadIdx.x >> 6), l = threadIdx.x & 63;
  if (g > a.groups) return;
  int* row = a.before + (long long)g * a.blocks;
  int done = 0;
  for (int b0 = 0; b0 < a.blocks; b0 += 64) {
    const int v = b0 + l < a.blocks ? row[b0 + l] : 0;
    const int upto = wave_scan_add(v);
    if (b0 + l < a.blocks) row[b0 + l] = done + upto - v;
    done += __shfl(upto, 63);
  }
  if (l == 0) a.all[g] = done;
}

// How a block knows what the others have: it is the only one; it adds up their counts itself (up to 64 blocks of up to 64 labels, the launch of sort_scan_kernel less); or that has been done.
enum Others { ONE, FUSED, SCANNED };

// WAVES waves with EACH labels a lane.
template <int WAVES, int EACH, Others O>
__global__ __launch_bounds__(64 * WAVES) void sort_place_kernel(SortArgs a) {
  extern __shared__ int lds[];
  __shared__ int part[WAVES];
  const int labels = a.groups + 1, wave = threadIdx.x >> 6, l = threadIdx.x & 63;
  int* first = lds;                                               // [labels]: where a label's begin
  int* mine = lds + labels + wave * labels;                       // [labels] of the wave: counts, then where its next one goes
  int* ahead = lds + labels * (WAVES + 1);                        // [labels] (FUSED): of the blocks before
  const int begin = blockIdx.x * (WAVES * EACH * 64) + wave * (EACH * 64) + l;
  int g[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) g[j] = begin + j * 64 < a.n ? label_of(a, begin + j * 64) : -1;
  for (int i = threadIdx.x; i < labels * (WAVES + 1); i += 64 * WAVES) lds[i] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j)
    if (g[j] >= 0) atomicAdd(&mine[g[j]], 1);
  if constexpr (O == FUSED) {
    for (int i = wave; i < labels; i += WAVES) {
      const int v = l < a.blocks ? a.before[(long long)i * a.blocks + l] : 0, upto = wave_scan_add(v);
      const int total = __shfl(upto, 63), less = __shfl(upto - v, blockIdx.x);
      if (l == 0) {
        first[i] = total;
        ahead[i] = less;
      }
    }
  }
  __syncthreads();
  if constexpr (O != FUSED) {
    for (int i = threadIdx.x; i < labels; i += 64 * WAVES) {
      int t = 0;
      if (O == ONE)
#pragma unroll
        for (int w = 1; w <= WAVES; ++w) t += lds[w * labels + i];
      first[i] = O == ONE ? t : a.all[i];
    }
    __syncthreads();
  }
  // an exclusive sum over the labels, a stretch of them a thread
  const int per = (labels + 64 * WAVES - 1) / (64 * WAVES), g0 = min(labels, (int)threadIdx.x * per), g1 = min(labels, g0 + per);
  int sum = 0;
  for (int i = g0; i < g1; ++i) sum += first[i];
  const int upto = wave_scan_add(sum);
  if (l == 63) part[wave] = upto;
  __syncthreads();
  int at = upto - sum;
  for (int w = 0; w < wave; ++w) at += part[w];
  for (int i = g0; i < g1; ++i) {
    int t = at;
    at += first[i];
    if (blockIdx.x == 0) a.offs[i] = t;
    if (O == FUSED) t += ahead[i];
    if (O == SCANNED) t += a.before[(long long)i * a.blocks + blockIdx.x];
#pragma unroll
    for (int w = 1; w <= WAVES; ++w) {
      const int n = lds[w * labels + i];
      lds[w * labels + i] = t;
      t += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const bool in = g[j] >= 0;
    // the lanes with this lane's label
    unsigned long long same = __ballot(in);
    if (!same) break;
    for (int b = 0; b < a.bits; ++b) {
      const unsigned long long set = __ballot(g[j] >> b & 1);
      same &= g[j] >> b & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << l) - 1)), leader = in ? __ffsll((unsigned long long)same) - 1 : l;
    int base = 0;
    if (in && l == leader) base = atomicAdd(&mine[g[j]], __popcll(same));
    const int to = __shfl(base, leader) + rank, i = begin + j * 64;
    if (in) {
      if (a.place) a.place[i] = to;
      if (a.order) a.order[to] = i;
    }
  }
}

// ---- rows ----

struct RowsArgs {
  const void *x, *residual;
  void* y;
  const int *place, *offs;
  const float* weight;
  long long x_stride, residual_stride, y_stride;
  RowChunks s;
  int cols, k, groups, n;                                         // n: rows * k
};

constexpr int ROW_TILE = 256;

// How many places are experts' (the rest are of none).
__device__ __forceinline__ int routed_of(const int* offs, int groups, int n) { return min(max(offs[groups], 0), n); }

constexpr int AT_ONCE = 4;                                        // choices whose rows are in flight together

// The block's turns over all chunks: row and first column of this thread's in each, and how many columns are left.
template <typename F>
__device__ __forceinline__ void each_chunk(const RowChunks& s, int cols, F&& go) {
  const long long chunks = s.rows * s.eights;
  for (long long first = (long long)blockIdx.x * ROW_TILE; first < chunks; first += (long long)gridDim.x * ROW_TILE) {
    const long long row0 = first / s.eights;
    long long row;
    unsigned chunk;
    chunk_at(s, row0, (unsigned)(first - row0 * s.eights), threadIdx.x, row, chunk);
    if (first + threadIdx.x < chunks) go(row, (int)chunk * 8, cols - (int)chunk * 8);
  }
}

template <typename T, bool VEC, bool PAST>
__global__ __launch_bounds__(256) void gather_kernel(RowsArgs a) {
  const int routed = routed_of(a.offs, a.groups, a.n);
  each_chunk(a.s, a.cols, [&](long long row, int col, int left) {
    Raw8<T> v, none;
    v.template load<VEC>((const T*)a.x + row * a.x_stride + col, left);
#pragma unroll
    for (unsigned& w : none.w) w = 0;
    for (int s0 = 0; s0 < a.k; s0 += AT_ONCE) {
      int p[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) p[j] = s0 + j < a.k ? a.place[row * a.k + s0 + j] : -1;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        T* to = (T*)a.y + p[j] * a.y_stride + col;
        if ((unsigned)p[j] < (unsigned)routed) v.template store<VEC, PAST>(to, left);
        else if ((unsigned)p[j] < (unsigned)a.n) none.template store<VEC, PAST>(to, left);
      }
    }
  });
}

template <typename T, bool VEC, bool PAST>
__global__ __launch_bounds__(256) void combine_kernel(RowsArgs a) {
  const int routed = routed_of(a.offs, a.groups, a.n);
  each_chunk(a.s, a.cols, [&](long long row, int col, int left) {
    Raw8<T> res;
    if (a.residual) res.template load<VEC>((const T*)a.residual + row * a.residual_stride + col, left);
    float v[8] = {};
    for (int s0 = 0; s0 < a.k; s0 += AT_ONCE) {
      int p[AT_ONCE];
      float w[AT_ONCE];
      Raw8<T> out[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        p[j] = s0 + j < a.k ? a.place[row * a.k + s0 + j] : -1;
        w[j] = s0 + j < a.k && a.weight ? a.weight[row * a.k + s0 + j] : 1.f;
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if ((unsigned)p[j] < (unsigned)routed) out[j].template load<VEC>((const T*)a.x + p[j] * a.x_stride + col, left);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if ((unsigned)p[j] < (unsigned)routed) {
          float o[8];
          out[j].values(o);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += w[j] * o[i];
        }
    }
    if (a.residual) {
      float r[8];
      res.values(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store8<T, VEC, PAST>((T*)a.y + row * a.y_stride + col, left, v);
  });
}

struct CombineBackArgs {
  const void *dy, *out;
  void* dout;
  const int *place, *offs;
  const float* weight;
  float* dweight;
  long long dy_stride, out_stride, dout_stride, rows;
  int cols, k, groups, n;
};

// WAVES waves a row (blocks of four waves), four choices at a time.  DOTS: with dweight, for which alone `out` is read (16384 x 4096 to two in bf16 122 us, without 59; 1117 x 1000 to three in
// fp32 7.3, 6.2; with the question in the kernel 2000 x 2048 to two took 9.0 us for 8.4).
template <typename T, int WAVES, bool VEC, bool PAST, bool DOTS>
__global__ __launch_bounds__(256) void combine_back_kernel(CombineBackArgs a) {
  __shared__ float part[4][AT_ONCE];
  constexpr int ROWS = 4 / WAVES;
  const int routed = routed_of(a.offs, a.groups, a.n), wave = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int lane = WAVES == 1 ? l : threadIdx.x;
  for (long long row0 = (long long)blockIdx.x * ROWS; row0 < a.rows; row0 += (long long)gridDim.x * ROWS) {
    const long long row = row0 + (WAVES == 1 ? wave : 0);
    const bool in = row < a.rows;
    for (int s0 = 0; s0 < a.k; s0 += AT_ONCE) {
      int p[AT_ONCE];
      float w[AT_ONCE], dot[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const bool is = in && s0 + j < a.k;
        p[j] = is ? a.place[row * a.k + s0 + j] : -1;
        w[j] = is && a.weight ? a.weight[row * a.k + s0 + j] : 1.f;
        dot[j] = 0.f;
      }
      if (in)
        for (int col = lane * 8; col < a.cols; col += 64 * WAVES * 8) {
          const int left = a.cols - col;
          Raw8<T> raw, out[AT_ONCE];
          raw.template load<VEC>((const T*)a.dy + row * a.dy_stride + col, left);
#pragma unroll
          for (int j = 0; j < AT_ONCE; ++j)
            if (DOTS && (unsigned)p[j] < (unsigned)routed) out[j].template load<VEC>((const T*)a.out + p[j] * a.out_stride + col, left);
          float d[8];
          raw.values(d);
#pragma unroll
          for (int j = 0; j < AT_ONCE; ++j) {
            if ((unsigned)p[j] >= (unsigned)a.n) continue;
            float o[8] = {};
            if (p[j] < routed) {
              if constexpr (DOTS) out[j].values(o);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                if constexpr (DOTS) dot[j] += d[i] * o[i];
                o[i] = w[j] * d[i];
              }
            }
            if (a.dout) store8<T, VEC, PAST>((T*)a.dout + p[j] * a.dout_stride + col, left, o);
          }
        }
      if constexpr (!DOTS) continue;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
        for (int x = 1; x < 64; x *= 2) dot[j] += __shfl_xor(dot[j], x);
      if (WAVES > 1) {
        __syncthreads();
        if (l < AT_ONCE) part[wave][l] = l == 0 ? dot[0] : l == 1 ? dot[1] : l == 2 ? dot[2] : dot[3];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) dot[j] = part[0][j] + part[1][j] + part[2][j] + part[3][j];
      }
      if (in && lane < AT_ONCE && s0 + lane < a.k)
        a.dweight[row * a.k + s0 + lane] = lane == 0 ? dot[0] : lane == 1 ? dot[1] : lane == 2 ? dot[2] : dot[3];
    }
  }
}

int sort_blocks(long long n) { return (int)((n + STRETCH - 1) / STRETCH); }
// Labels that one block sorts in a launch: sixteen waves of 256 each, where their counts fit into LDS (3351 labels of ten groups: 6.1 us, in three launches 12.8).
int sort_at_once(int groups) { return groups <= 512 ? 4096 : STRETCH; }

gan_status check_exchange(int32_t precision, int64_t rows, int32_t cols, int32_t groups, int32_t k) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if (groups < 0 || k < 1) return operator_fail(GAN_E_ARG, "negative groups, or no choices");
  if (groups > 65535 || k > MOST_ROWS || rows * k > MOST_ROWS) return operator_fail(GAN_E_SHAPE, "more than 65535 groups or 2^30 choices");
  return GAN_OK;
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" int64_t gan_sort_by_label_bytes(int64_t n, int32_t groups) {
  if (n > MOST_ROWS || groups < 0 || groups > MOST_LABELS || n <= sort_at_once(groups)) return 0;
  return ((int64_t)sort_blocks(n) + 1) * (groups + 1) * 4;
}

extern "C" gan_status gan_sort_by_label(const int32_t* labels, int64_t n, int32_t groups, int32_t* offs, int32_t* order, int32_t* place, void* work, int64_t work_bytes,
                                        void* hip_stream) {
  if (n < 0 || groups < 0) return operator_fail(GAN_E_ARG, "negative n or groups");
  if (n > MOST_ROWS || groups > MOST_LABELS) return operator_fail(GAN_E_SHAPE, "more than 2^30 labels or 4096 groups");
  if ((n > 0 && !labels) || !offs) return operator_fail(GAN_E_ARG, "labels or offs is NULL");
  const int64_t need = gan_sort_by_label_bytes(n, groups);
  if (work_bytes < need || (need > 0 && !work) || !aligned16(work)) return operator_fail(GAN_E_ARG, "work is smaller than gan_sort_by_label_bytes, or not 16-byte aligned");
  operator_launches();
  const hipStream_t st = (hipStream_t)hip_stream;
  int bits = 0;
  while (groups >> bits) ++bits;
  const int blocks = sort_blocks(n), labels_all = groups + 1;
  const SortArgs a = {labels, offs, order, place, (int*)work, (int*)work + (long long)blocks * labels_all, (int)n, groups, blocks, bits};
  const unsigned one = labels_all * 4;
  if (need == 0) {
    if (groups <= 512) hipLaunchKernelGGL((sort_place_kernel<16, 4, ONE>), dim3(1), dim3(1024), 17 * one, st, a);
    else if (groups <= 2048) hipLaunchKernelGGL((sort_place_kernel<4, 8, ONE>), dim3(1), dim3(256), 5 * one, st, a);
    else hipLaunchKernelGGL((sort_place_kernel<2, 16, ONE>), dim3(1), dim3(128), 3 * one, st, a);
    return operator_launched();
  }
  const bool fused = blocks <= 64 && groups < 64;
  hipLaunchKernelGGL(sort_count_kernel, dim3(blocks), dim3(1024), one, st, a);
  if (!fused) hipLaunchKernelGGL(sort_scan_kernel, dim3((labels_all + 3) / 4), dim3(256), 0, st, a);
  if (fused) hipLaunchKernelGGL((sort_place_kernel<16, 2, FUSED>), dim3(blocks), dim3(1024), 18 * one, st, a);
  else if (groups <= 512) hipLaunchKernelGGL((sort_place_kernel<16, 2, SCANNED>), dim3(blocks), dim3(1024), 17 * one, st, a);
  else if (groups <= 2048) hipLaunchKernelGGL((sort_place_kernel<4, 8, SCANNED>), dim3(blocks), dim3(256), 5 * one, st, a);
  else hipLaunchKernelGGL((sort_place_kernel<2, 16, SCANNED>), dim3(blocks), dim3(128), 3 * one, st, a);
  return operator_launched();
}

extern "C" gan_status gan_gather_rows(int32_t precision, const void* x, int64_t x_stride, const int32_t* place, const int32_t* offs, int32_t groups, int32_t k, int64_t rows,
                                      int32_t cols, void* out, int64_t out_stride, void* hip_stream) {
  if (const gan_status s = check_exchange(precision, rows, cols, groups, k)) return s;
  if (!offs || (rows > 0 && (!x || !place || !out))) return operator_fail(GAN_E_ARG, "x, place, offs or out is NULL");
  for (const gan_status s : {check_matrix(x, x_stride, cols, "x_stride is below cols"), check_matrix(out, out_stride, cols, "out_stride is below cols")})
    if (s) return s;
  if (rows == 0) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % 8 == 0 && rows_aligned16(x, x_stride, e) && rows_aligned16(out, out_stride, e);
  const RowsArgs a = {x, nullptr, out, place, offs, nullptr, x_stride, 0, out_stride, row_chunks(rows, cols), cols, k, groups, (int)(rows * k)};
  const dim3 grid(chunk_blocks(a.s, ROW_TILE, 1 << 20));
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool past = rows * k * cols * e > PAST_CACHES;
#define GAN_GATHER(T, V) \
  if (V && past) hipLaunchKernelGGL((gather_kernel<T, V, V>), grid, dim3(256), 0, st, a); \
  else hipLaunchKernelGGL((gather_kernel<T, V, false>), grid, dim3(256), 0, st, a)
  if (precision == GAN_FP32) { if (vec) { GAN_GATHER(float, true); } else { GAN_GATHER(float, false); } }
  else { if (vec) { GAN_GATHER(bf16_t, true); } else { GAN_GATHER(bf16_t, false); } }
#undef GAN_GATHER
  return operator_launched();
}

extern "C" gan_status gan_combine_rows(int32_t precision, const void* out, int64_t out_stride, const int32_t* place, const float* weight, const int32_t* offs, int32_t groups,
                                       int32_t k, const void* residual, int64_t residual_stride, int64_t rows, int32_t cols, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check_exchange(precision, rows, cols, groups, k)) return s;
  if (!offs || (rows > 0 && (!out || !place || !y))) return operator_fail(GAN_E_ARG, "out, place, offs or y is NULL");
  for (const gan_status s : {check_matrix(out, out_stride, cols, "out_stride is below cols"), check_matrix(residual, residual_stride, cols, "residual_stride is below cols"),
                             check_matrix(y, y_stride, cols, "y_stride is below cols")})
    if (s) return s;
  if (rows == 0) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % 8 == 0 && rows_aligned16(out, out_stride, e) && (!residual || rows_aligned16(residual, residual_stride, e)) && rows_aligned16(y, y_stride, e);
  const RowsArgs a = {out, residual, y, place, offs, weight, out_stride, residual_stride, y_stride, row_chunks(rows, cols), cols, k, groups, (int)(rows * k)};
  const dim3 grid(chunk_blocks(a.s, ROW_TILE, 1 << 20));
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool past = rows * cols * e > PAST_CACHES;
#define GAN_COMBINE(T, V) \
  if (V && past) hipLaunchKernelGGL((combine_kernel<T, V, V>), grid, dim3(256), 0, st, a); \
  else hipLaunchKernelGGL((combine_kernel<T, V, false>), grid, dim3(256), 0, st, a)
  if (precision == GAN_FP32) { if (vec) { GAN_COMBINE(float, true); } else { GAN_COMBINE(float, false); } }
  else { if (vec) { GAN_COMBINE(bf16_t, true); } else { GAN_COMBINE(bf16_t, false); } }
#undef GAN_COMBINE
  return operator_launched();
}

extern "C" gan_status gan_combine_rows_backward(int32_t precision, const void* dy, int64_t dy_stride, const void* out, int64_t out_stride, const int32_t* place,
                                                const float* weight, const int32_t* offs, int32_t groups, int32_t k, int64_t rows, int32_t cols, void* dout, int64_t dout_stride,
                                                float* dweight, void* hip_stream) {
  if (const gan_status s = check_exchange(precision, rows, cols, groups, k)) return s;
  if (!offs || (rows > 0 && (!dy || !place))) return operator_fail(GAN_E_ARG, "dy, place or offs is NULL");
  if (rows > 0 && dweight && !out) return operator_fail(GAN_E_ARG, "out, which dweight is made of, is NULL");
  for (const gan_status s : {check_matrix(dy, dy_stride, cols, "dy_stride is below cols"), check_matrix(out, out_stride, cols, "out_stride is below cols"),
                             check_matrix(dout, dout_stride, cols, "dout_stride is below cols")})
    if (s) return s;
  if (rows == 0 || (!dout && !dweight)) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % 8 == 0 && rows_aligned16(dy, dy_stride, e) && (!dweight || rows_aligned16(out, out_stride, e)) && (!dout || rows_aligned16(dout, dout_stride, e));
  const CombineBackArgs a = {dy, out, dout, place, offs, weight, dweight, dy_stride, out_stride, dout_stride, rows, cols, k, groups, (int)(rows * k)};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool wide = cols > 1024;
  const dim3 grid((unsigned)std::min(wide ? (long long)rows : ((long long)rows + 3) / 4, 1ll << 20));
  // (In fp32 without dweight they go through the caches: nothing is read between a lane's two stores of a row, and past the caches these reach memory as half lines.  us through and past,
  // 8192 x 1024 to four: 29, 65; 16384 x 2048 to two: 76, 105; with dweight 58, 55 and 128, 139; bf16 without, 16384 x 4096 to two: 72, 59.)
  const bool past = rows * k * cols * e > PAST_CACHES;
#define GAN_COMBINE_BACK(T, W, V) \
  if (dweight && V && past) hipLaunchKernelGGL((combine_back_kernel<T, W, V, V, true>), grid, dim3(256), 0, st, a); \
  else if (dweight) hipLaunchKernelGGL((combine_back_kernel<T, W, V, false, true>), grid, dim3(256), 0, st, a); \
  else if (V && past && sizeof(T) == 2) hipLaunchKernelGGL((combine_back_kernel<T, W, V, V && sizeof(T) == 2, false>), grid, dim3(256), 0, st, a); \
  else hipLaunchKernelGGL((combine_back_kernel<T, W, V, false, false>), grid, dim3(256), 0, st, a)
  if (precision == GAN_FP32) {
    if (wide) { if (vec) { GAN_COMBINE_BACK(float, 4, true); } else { GAN_COMBINE_BACK(float, 4, false); } }
    else { if (vec) { GAN_COMBINE_BACK(float, 1, true); } else { GAN_COMBINE_BACK(float, 1, false); } }
  } else {
    if (wide) { if (vec) { GAN_COMBINE_BACK(bf16_t, 4, true); } else { GAN_COMBINE_BACK(bf16_t, 4, false); } }
    else { if (vec) { GAN_COMBINE_BACK(bf16_t, 1, true); } else { GAN_COMBINE_BACK(bf16_t, 1, false); } }
  }
#undef GAN_COMBINE_BACK
  return operator_launched();
}
