// Matrix products grouped by label: every expert's rows times its own weights, the gradient of the rows, and that of the weights; in fp32,
// bf16 and 8 bits.
//
//   forward   y[i]  = w[g] x[i]              C(m, n) = sum_k A(m, k) B(n, k):   A = x,  B = w[g],  k = inputs
//   dgrad     dx[i] = dy[i] w[g]                                                A = dy, B = w[g]^T, k = outputs
//   wgrad     dw[g] = sum of dy[i]^T x[i]                                       A = dy^T, B = x^T, k = g's rows
//
// "k-major" below: the sum's index runs along memory (both operands of the forward product, dy of dgrad); the others have it as the row.
// Which expert a tile of rows belongs to every wave finds itself from the offsets, so that a call is one launch.
//
// Times on an MI355X (its library's product of 8192^3: 1.36 PFLOP/s in bf16; a copy: 4.9 TB/s).  bf16 tiles: 8192^3 as one expert 1.24-1.35 PFLOP/s, forward, dgrad and wgrad, 1.33
// from 8 bits: bound by the matrix pipe and the clock that its power leaves (its share of the cycles at eight experts of 2048 rows, 4096 -> 4096: 0.57, 0.54 from 8 bits).  Of the cycles
// of LDS 3 % are bank conflicts, all from the stores of the results, and 29 % from 8 bits, where the converted operands are stored too.  With drawn sizes of 2048 rows on average
// 480-500 us, where the experts' last tiles cost a tenth (equal experts: 454), and 447-472 from 8 bits (439); weight gradient 493-509, of which
// 537 MB of fp32 results are 110.  A hundred experts of unequal sizes, 1024 -> 1024, cold weights: 57 us forward, 49 dgrad, 96 wgrad (4.7 TB/s): bound by the
// weights' bytes.  Few rows: ten rows of a hundred experts 7 us (21 MB of weights), eight of eight experts in 8 bits 27-29 us (90 MB).
#include "code_walk.h"
#include "group_tiles.h"
#include "lds_copy.h"
#include "operators.h"
#include "split_mfma.h"

#include <algorithm>

namespace gan {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

enum Kind { FORWARD = 0, DGRAD = 1, WGRAD = 2 };

struct LinearArgs {
  const void *a, *b;             // as above; b: expert 0's
  const uint8_t *a_scale, *b_scale;
  void* c;
  const int* offs;
  long long a_stride, b_stride, c_stride;      // of memory rows, in elements
  long long b_group, c_group;                  // between experts (c_group: wgrad)
  int groups, rows;
  int m, n, k;                                 // wgrad: m = outputs, n = inputs; else n, k (m: the expert's rows; wgrad: k)
  int parts;                                   // wgrad: an expert's rows are shared by this many blocks, whose results follow one another at `part` elements
  long long part;
  unsigned first;                              // of the launch's tiles among the call's
};

// The block's number among all of the call's.
__device__ __forceinline__ unsigned block_of(const LinearArgs& q) { return q.first + blockIdx.x; }

// ---- fp32 ----
//
// Bound by the matrix pipe, which six bf16 products a value keep busy, and the vector instructions that split the operands: eight experts of 1024 rows on average, 2048 -> 2048,
// 459 us forward, 447 dgrad, 377 wgrad = 150-182 TFLOP/s (equal experts 388, 376, 373; the library's fp32 product: 133 TFLOP/s).
// RT x RT tiles (128 or 64), 32 of the sum's index at a time: loaded into registers while the last ones are multiplied, then written to LDS as three planes of bf16
// parts (split_mfma.h).  What has the sum's index as its row is kept that way and read with transposing LDS reads.
constexpr int RK = 32;

template <bool KMAJOR, int RT>
struct Staged {
  static constexpr int PLANE = RT * RK * 2, CHUNKS = RT / 64, PER_ROW = KMAJOR ? RK / 8 : RT / 8;
  float v[CHUNKS][8];

  // thread t's chunks of eight: k-major row t / 4 (+ 64), elements 8 (t % 4) ..; else sum index t / PER_ROW (+ 16), columns 8 (t % PER_ROW) ..
  __device__ static __forceinline__ int row_of(int h) { return (threadIdx.x + h * 256) / PER_ROW; }
  __device__ __forceinline__ void load(const float* p, long long stride, int row0, int rows, int k0, int k_end) {
#pragma unroll
    for (int h = 0; h < CHUNKS; ++h) {
      const int r = (KMAJOR ? row0 : k0) + row_of(h), c = (KMAJOR ? k0 : row0) + threadIdx.x % PER_ROW * 8;
      const int left = r < (KMAJOR ? rows : k_end) ? (KMAJOR ? k_end : rows) - c : 0;
      load8<float, false>(p + (long long)r * stride + c, left, v[h]);
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int h = 0; h < CHUNKS; ++h) {
      unsigned char* at = lds + offset(row_of(h), threadIdx.x % PER_ROW);
      u32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __float_as_uint(v[h][i]);
        hi[i] = __float_as_uint(v[h][4 + i]);
      }
      const Split8 s = split8(lo, hi);
      *reinterpret_cast<u32x4*>(at) = s.h;
      *reinterpret_cast<u32x4*>(at + PLANE) = s.m;
      *reinterpret_cast<u32x4*>(at + 2 * PLANE) = s.l;
    }
  }
  // Granules of eight elements are exchanged within a row so that the lanes of a read fall into different banks: rows of 64 bytes (k-major), read
  // sixteen rows at a time, and of 256 or 128, read with eight sum indices at a time.
  __device__ static __forceinline__ int swap_of(int r) {
    if constexpr (KMAJOR) return (r >> 2) & 3;
    else if constexpr (PER_ROW >= 16) return ((r & 3) | ((r >> 3) & 1) << 2) << 1;
    else return (((r >> 1) & 1) | ((r >> 3) & 1) << 1) << 1;
  }
  __device__ static __forceinline__ int offset(int r, int granule) { return r * (PER_ROW * 16) + (granule ^ swap_of(r)) * 16; }

  // the MFMA operand of rows row .. row + 15: lane l has row l % 16, sum indices 8 (l / 16) .. + 7
  __device__ static __forceinline__ u32x4 read(const unsigned char* lds, int row) {
    const int l = threadIdx.x & 63;
    if constexpr (KMAJOR) {
      return *reinterpret_cast<const u32x4*>(lds + offset(row + (l & 15), l >> 4));
    } else {
      const int k = (l >> 4) * 8 + ((l & 15) >> 2);
      const uint2 a = lds_read_tr16(lds + offset(k, row / 8 + ((l & 3) >> 1)) + (l & 1) * 8);
      const uint2 b = lds_read_tr16(lds + offset(k + 4, row / 8 + ((l & 3) >> 1)) + (l & 1) * 8);
      return u32x4{a.x, a.y, b.x, b.y};
    }
  }
};

__device__ __forceinline__ void mma(floatx4& acc, const u32x4& a, const u32x4& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}

// four neighbouring outputs of one row, of any alignment
template <typename C>
__device__ __forceinline__ void store_four(C* p, int left, const float (&v)[4]) {
  if (left >= 4) {
    if constexpr (sizeof(C) == 4) {
      *reinterpret_cast<Words<4>::T*>(p) = Words<4>::T{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
      typedef unsigned two __attribute__((ext_vector_type(2), aligned(2)));
      *reinterpret_cast<two*>(p) = two{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = from_float<C>(v[i]);
  }
}

// The part of an expert's rows that block `part` of `parts` takes: whole steps of 64.
__device__ __forceinline__ void part_of(int part, int parts, int& begin, int& end) {
  const int each = ((end - begin + parts - 1) / parts + 63) / 64 * 64;
  begin = (int)min((long long)begin + (long long)part * each, (long long)end);
  end = min(end - begin, each) + begin;
}

// A wave's outputs, rows m .. (of m_end) and columns n .. (of n_end), as MFMAs with the columns first leave them.  Sixteen rows at a time go through LDS (the wave's
// own), so that its lanes store whole rows, 16 bytes each: 64 lanes with four columns each of sixteen rows would write 32 or 64 bytes of a row at a time (the weight
// gradient of a hundred experts of 1024 x 1024: 173 us, 125 by rows).
// PAST: past the caches.  A weight gradient's results are more than what they are made of and push it out of them (a hundred experts of 1024 x 1024: 124 us, 92 past
// the caches; eight of 4096 x 4096: 527, 493; ten of 512 x 784: 11, 9.3; followed by the AdamW step that reads them, 8-bit moments, a hundred of 1024 x 1024 447, 435, ten of 512 x 784
// 29.2, 28.0, with 32-bit moments 33.1, 33.7).  The partial sums of a split gradient, which sum_parts_kernel reads next, go the same way, though they would be faster through the caches (both
// launches, bf16, one expert of 16384 rows: 512 x 512 34, past them 38; 128 x 128 24, 33).  A layer's outputs are read next, and stay.
template <typename C, bool PAST, int TM, int TN>
__device__ __forceinline__ void store_rows(const floatx4 (&acc)[TM][TN], C* c, long long stride, unsigned char* lds, int m0, int m_end, int n0, int n_end) {
  constexpr int WIDE = TN * 16 * (int)sizeof(C), LANES = WIDE / 16, EACH = 16 / (int)sizeof(C);
  static_assert(64 % LANES == 0, "whole rows");
  typedef typename Words<sizeof(C)>::T words;
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if (m0 + i * 16 >= m_end) break;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      unsigned char* at = lds + (l & 15) * (WIDE + 16) + (j * 16 + (l >> 4) * 4) * (int)sizeof(C);
      if constexpr (sizeof(C) == 4) *reinterpret_cast<floatx4*>(at) = acc[i][j];
      else *reinterpret_cast<uint2*>(at) = make_uint2(pack2_bf16(acc[i][j][0], acc[i][j][1]), pack2_bf16(acc[i][j][2], acc[i][j][3]));
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = l / LANES; r < 16; r += 64 / LANES) {
      const int m = m0 + i * 16 + r, n = n0 + l % LANES * EACH;
      const unsigned char* from = lds + r * (WIDE + 16) + l % LANES * 16;
      const uint4 v = *reinterpret_cast<const uint4*>(from);
      if (m >= m_end || n >= n_end) continue;
      C* at = c + (long long)m * stride + n;
      if (n + EACH <= n_end) {
        const words o = {v.x, v.y, v.z, v.w};
        if constexpr (PAST) __builtin_nontemporal_store(o, reinterpret_cast<words*>(at));
        else *reinterpret_cast<words*>(at) = o;
      } else {
        for (int k = 0; k < n_end - n; ++k) at[k] = reinterpret_cast<const C*>(from)[k];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int KIND, int RT>
__global__ __launch_bounds__(256, RT == 128 ? 2 : 4) void linear_fp32_kernel(LinearArgs q) {
  typedef Staged<KIND != WGRAD, RT> SA;
  typedef Staged<KIND == FORWARD, RT> SB;
  constexpr int TW = RT / 32;                                     // sixteens of a wave's rows, and of its columns
  __shared__ __align__(16) unsigned char lds[2 * 3 * RT * RK * 2];
  unsigned char *la = lds, *lb = lds + 3 * RT * RK * 2;

  const unsigned block = block_of(q);
  const int n_tiles = (q.n + RT - 1) / RT, n0 = (int)(block % n_tiles) * RT;
  int group, m0, m_end, k_begin = 0, k_end = q.k, part = 0;
  if (KIND == WGRAD) {
    const int m_tiles = (q.m + RT - 1) / RT, t = block / n_tiles, e = t / m_tiles;
    part = e % q.parts;
    group = e / q.parts;
    m0 = t % m_tiles * RT;
    m_end = q.m;
    group_rows(q.offs, q.groups, q.rows, group, k_begin, k_end);
    part_of(part, q.parts, k_begin, k_end);
  } else {
    if (!find_tile(q.offs, q.groups, q.rows, RT, block / n_tiles, group, m0, m_end)) return;
    if (group == q.groups) k_end = 0;                             // rows of no expert: zeros
  }
  const float* a = (const float*)q.a;
  const float* b = (const float*)q.b + (KIND == WGRAD ? 0 : (long long)(group < q.groups ? group : 0) * q.b_group);
  float* c = (float*)q.c + (KIND == WGRAD ? part * q.part + (long long)group * q.c_group : 0);

  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, wm = (wave >> 1) * (RT / 2), wn = (wave & 1) * (RT / 2);
  floatx4 acc[TW][TW], low[TW][TW];
#pragma unroll
  for (int i = 0; i < TW; ++i)
#pragma unroll
    for (int j = 0; j < TW; ++j) acc[i][j] = low[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  SA sa;
  SB sb;
  if (k_begin < k_end) {
    sa.load(a, q.a_stride, m0, m_end, k_begin, k_end);
    sb.load(b, q.b_stride, n0, q.n, k_begin, k_end);
  }
  for (int k0 = k_begin; k0 < k_end; k0 += RK) {
    __syncthreads();
    sa.store(la);
    sb.store(lb);
    __syncthreads();
    if (k0 + RK < k_end) {
      sa.load(a, q.a_stride, m0, m_end, k0 + RK, k_end);
      sb.load(b, q.b_stride, n0, q.n, k0 + RK, k_end);
    }
    u32x4 fa[TW][3];
#pragma unroll
    for (int i = 0; i < TW; ++i)
#pragma unroll
      for (int p = 0; p < 3; ++p) fa[i][p] = SA::read(la + p * SA::PLANE, wm + i * 16);
#pragma unroll
    for (int j = 0; j < TW; ++j) {
      u32x4 fb[3];
#pragma unroll
      for (int p = 0; p < 3; ++p) fb[p] = SB::read(lb + p * SB::PLANE, wn + j * 16);
#pragma unroll
      for (int i = 0; i < TW; ++i) {                               // (b first: a lane then holds four neighbouring columns of one row)
        mma(acc[i][j], fb[0], fa[i][0]);
        mma(low[i][j], fb[0], fa[i][1]);
        mma(low[i][j], fb[1], fa[i][0]);
        mma(low[i][j], fb[1], fa[i][1]);
        mma(low[i][j], fb[0], fa[i][2]);
        mma(low[i][j], fb[2], fa[i][0]);
      }
    }
  }

  bool again = false;
#pragma unroll
  for (int i = 0; i < TW; ++i)
#pragma unroll
    for (int j = 0; j < TW; ++j) {
      acc[i][j] = (acc[i][j] + low[i][j]) * SPLIT_UNSCALE;
#pragma unroll
      for (int e = 0; e < 4; ++e) again |= !finite_bits(__float_as_uint(acc[i][j][e]) & 0x7fffffffu);
    }
  // Infinities, NaN and what is out of the parts' range (values from 2^104, sums from 2^80) leave outputs that are not finite: a wave that has one sums its tile again with the
  // fp32 MFMAs, straight from memory, and takes those outputs from there.  Finite ones stay: a row's results do not depend on its neighbours'.  Eight experts of 1024 rows,
  // 2048 -> 2048, with one NaN / of NaN alone: 613 / 2121 us forward, 610 / 1402 dgrad, 465 / 1035 wgrad, of finite values 408, 447, 412 (each lane by chains of its own: 8331 / 61220, 13879 / 68474, 12535 / 71471).
  if (__any(again)) {
    floatx4 sum[TW][TW];
#pragma unroll
    for (int i = 0; i < TW; ++i)
#pragma unroll
      for (int j = 0; j < TW; ++j) sum[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = k_begin; k0 < k_end; k0 += 16) {
      float fa[4][TW], fb[4][TW];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int k = k0 + (l >> 4) * 4 + e;
#pragma unroll
        for (int i = 0; i < TW; ++i) {
          const int m = m0 + wm + i * 16 + (l & 15), n = n0 + wn + i * 16 + (l & 15);
          fa[e][i] = k < k_end && m < m_end ? KIND == WGRAD ? a[(long long)k * q.a_stride + m] : a[(long long)m * q.a_stride + k] : 0.f;
          fb[e][i] = k < k_end && n < q.n ? KIND == FORWARD ? b[(long long)n * q.b_stride + k] : b[(long long)k * q.b_stride + n] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < TW; ++j)
#pragma unroll
          for (int i = 0; i < TW; ++i) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[e][j], fa[e][i], sum[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < TW; ++i)
#pragma unroll
      for (int j = 0; j < TW; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!finite_bits(__float_as_uint(acc[i][j][e]) & 0x7fffffffu)) acc[i][j][e] = sum[i][j][e];
  }
  __syncthreads();
  store_rows<float, KIND == WGRAD, TW, TW>(acc, c, q.c_stride, lds + wave * 16 * (TW * 64 + 16), m0 + wm, m_end, n0 + wn, q.n);
}

// ---- bf16 and 8 bits ----
//
// Tiles of BM x BN, 64 of the sum's index a step, in LDS as bf16: k-major operands in rows of 128 bytes, the others as 64 rows (sum indices) of BM or BN
// values that are read with transposing reads.  bf16 operands are copied straight from memory while the step before the last is multiplied; those whose rows are
// no multiples of 16 bytes go through registers, and so do 8-bit ones, where a code times its block's power of two becomes the bf16 number that it is (but for
// the subnormal codes of E = -126 and -125, rounded to multiples of 2^-133, and values from 2^128 on, which are infinite): every product is exact and every sum fp32.
// (The 8-bit MFMAs would take half the matrix-pipe time, but they add eight neighbouring products with what lies 2^-13 below the largest of them
// cut off (2^16 + 2^2 is 2^16): 1.5e-5 of the result's norm on normal values, 5e-5 on codes of all sizes.)
constexpr int STEP = CODE_STEP;

// One operand's tile: R rows (or columns) of it, NW waves copying.
template <bool KMAJOR, int R, int NW>
struct Tile {
  static constexpr int BYTES = R * 128;
  static constexpr int PIECES = BYTES / 1024 / NW;                // of 1 KiB, for each wave
  static constexpr int PER_ROW = R / 8;                           // granules of a row that is no k-major one
  static_assert(BYTES % (1024 * NW) == 0, "whole pieces");

  // Banks: sixteen lanes read sixteen k-major rows of 128 bytes at a time, or 32 lanes eight sum indices with 32 bytes each.
  __device__ static __forceinline__ int swap_of(int r) {
    if constexpr (KMAJOR) return (r >> 1) & 7;
    else if constexpr (PER_ROW >= 16) return ((r & 3) | ((r >> 3) & 1) << 2) << 1;
    else return (((r >> 1) & 1) | ((r >> 3) & 1) << 1) << 1;
  }
  // MFMA operand of rows row .. row + 15 (a multiple of 16): half h of the step
  __device__ static __forceinline__ u32x4 read(const unsigned char* lds, int row, int h) {
    const int l = threadIdx.x & 63;
    if constexpr (KMAJOR) {
      const int r = l & 15;
      return *reinterpret_cast<const u32x4*>(lds + row * 128 + r * 128 + (((h * 4 + (l >> 4)) ^ swap_of(r)) * 16));
    } else {
      const int k = (l >> 4) * 8 + ((l & 15) >> 2), g = (row / 8 + ((l & 3) >> 1)) ^ swap_of(k);
      const int k4 = k + 4, g4 = (row / 8 + ((l & 3) >> 1)) ^ swap_of(k4);
      const uint2 a = lds_read_tr16(lds + (h * 32 + k) * (R * 2) + g * 16 + (l & 1) * 8);
      const uint2 b = lds_read_tr16(lds + (h * 32 + k4) * (R * 2) + g4 * 16 + (l & 1) * 8);
      return u32x4{a.x, a.y, b.x, b.y};
    }
  }
};

__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(unsigned long long)(__attribute__((address_space(3))) const void*)p; }

// Eight neighbouring bf16 values of any alignment, of which `n` are the row's last (more than eight, or none).  The last few of a row are read as the end of its
// last eight (a row of fewer than eight: one by one), and shifted when they are used, so that nothing is waited for between the loads.
__device__ __forceinline__ u32x4 load_last(const bf16_t* p, int n, bool short_row) {
  u32x4 v = {0, 0, 0, 0};
  if (short_row) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) v[i / 2] |= (unsigned)p[i].v << 16 * (i % 2);
  } else if (n > 0) {
    v = __builtin_bit_cast(u32x4, *reinterpret_cast<const Words<2>::T*>(p - max(8 - n, 0)));
  }
  return v;
}
__device__ __forceinline__ u32x4 shift_last(const u32x4& v, int n, bool short_row) {
  if (n >= 8 || short_row) return v;
  unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
  const int bits = 16 * (8 - n);                                  // 16 or more
  if (bits >= 64) {
    lo = bits < 128 ? hi >> (bits - 64) : 0;
    hi = 0;
  } else {
    lo = lo >> bits | hi << (64 - bits);
    hi >>= bits;
  }
  return u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

// A bf16 operand whose rows are multiples of 16 bytes: copies.
template <bool KMAJOR, int R, int NW>
struct Copied : Tile<KMAJOR, R, NW> {
  typedef Tile<KMAJOR, R, NW> S;
  typedef bf16_t T;
  static constexpr bool COPIES = true;
  unsigned off[S::PIECES];                                        // byte offset of the lane's granule in the step's memory
  int4v memory;
  const unsigned char* at;                                        // the next step's memory, what there is of it, and the way to the one behind
  long long bytes, move;

  // rows (k-major; else columns) row0 .. of expert `base`, of which `rows` exist, sum indices k0 .. k_end - 1; stride in elements
  __device__ __forceinline__ void prepare(const T* base, const uint8_t*, long long stride, int row0, int rows, int k0, int k_end, int wave) {
    const int l = threadIdx.x & 63;
    at = (const unsigned char*)(base + (KMAJOR ? row0 * stride + k0 : k0 * stride + row0));
    bytes = (KMAJOR ? (rows - 1) * stride + k_end - k0 : (k_end - k0 - 1) * stride + rows) * 2;
    move = KMAJOR ? STEP * 2 : STEP * 2 * stride;
#pragma unroll
    for (int p = 0; p < S::PIECES; ++p) {
      const int piece = wave * S::PIECES + p;
      const int r = KMAJOR ? piece * 8 + (l >> 3) : piece * (64 / S::PER_ROW) + l / S::PER_ROW;
      const int g = (KMAJOR ? l & 7 : l % S::PER_ROW) ^ S::swap_of(r);
      off[p] = (KMAJOR ? r : g * 8) < rows ? (unsigned)(r * stride * 2) + g * 16 : NO_ROW;
    }
  }
  __device__ __forceinline__ void next_step() {
    memory = make_rsrc(at, (unsigned long long)max(bytes, 0ll));
    at += move;
    bytes -= move;
  }
  // piece p of the step, whose first sum index is `left` before the end
  __device__ __forceinline__ void piece(int p, int wave, int left, unsigned char*, unsigned lds) {
    const int l = threadIdx.x & 63, piece = wave * S::PIECES + p;
    const int k = KMAJOR ? ((l & 7) ^ S::swap_of(piece * 8 + (l >> 3))) * 8 : piece * (64 / S::PER_ROW) + l / S::PER_ROW;
    load16_to_lds(memory, k < left ? off[p] : NO_ROW, 0, lds + piece * 1024);
  }
};

// A bf16 operand of any alignment: chunks of eight elements, which are written to LDS a step after they were asked for.  Rows and columns that are not there are
// others again (their products are not stored); sum indices that are not there are zero.
template <bool KMAJOR, int R, int NW>
struct Loaded : Tile<KMAJOR, R, NW> {
  typedef Tile<KMAJOR, R, NW> S;
  typedef bf16_t T;
  static constexpr bool COPIES = false;
  static constexpr int CHUNKS = R * 8 / (64 * NW), ROW_CHUNKS = KMAJOR ? 8 : S::PER_ROW;
  static constexpr int PIECES = CHUNKS;
  static_assert(R * 8 % (64 * NW) == 0 && 64 * NW % ROW_CHUNKS == 0, "whole chunks, and a thread's all at one place of their rows");
  u32x4 q[CHUNKS];
  const T* at[CHUNKS];                                            // of the step that is asked for next
  long long move;
  int left;                                                       // the sum indices from it on
  int column_tail;                                                // elements of the row from the chunk on (other than k-major; 8 or more: all)
  bool short_row;

  __device__ static __forceinline__ int thread() { return threadIdx.x & (64 * NW - 1); }      // among the waves of the operand
  __device__ static __forceinline__ int row_of(int p) { return (thread() + p * 64 * NW) / ROW_CHUNKS; }
  __device__ static __forceinline__ int granule() { return thread() % ROW_CHUNKS; }
  __device__ __forceinline__ void prepare(const T* base, const uint8_t*, long long stride, int row0, int rows, int k0, int k_end, int) {
    left = k_end - k0;
    short_row = (KMAJOR ? k_end : row0 + rows) < 8;
    move = KMAJOR ? STEP : STEP * stride;
    const int c = KMAJOR ? granule() * 8 : min(granule() * 8, (rows - 1) / 8 * 8);
    column_tail = KMAJOR ? 8 : rows - c;
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      at[p] = base + (KMAJOR ? (row0 + min(row_of(p), rows - 1)) * stride + k0 : (k0 + row_of(p)) * stride + row0) + c;
      if (!short_row) at[p] -= max(8 - column_tail, 0);
      ask(p);
    }
    step_on();
  }
  __device__ __forceinline__ void step_on() {
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) at[p] += move;
    left -= STEP;
  }
  __device__ __forceinline__ void ask(int p) {
    if constexpr (KMAJOR) q[p] = load_last(at[p], left - granule() * 8, short_row);
    else q[p] = load_last(at[p], row_of(p) < left ? short_row ? column_tail : 8 : 0, short_row);
  }
  __device__ __forceinline__ void next_step() {}
  __device__ __forceinline__ void piece(int p, int, int, unsigned char* lds, unsigned) {
    const int r = row_of(p), g = granule() ^ S::swap_of(r);
    *reinterpret_cast<u32x4*>(lds + r * (KMAJOR ? 128 : R * 2) + g * 16) = shift_last(q[p], KMAJOR ? left + STEP - granule() * 8 : column_tail, short_row);
    ask(p);
    if (p == CHUNKS - 1) step_on();
  }
};

// An 8-bit operand, k-major: chunks of sixteen codes of a row, thread t's being chunk t % 4 of rows t / 4, t / 4 + THREADS / 4, ...  A chunk is written to LDS two
// steps after it was asked for.
template <int R, int NW>
struct Converted : Tile<true, R, NW> {
  typedef Tile<true, R, NW> S;
  __device__ static __forceinline__ int thread() { return threadIdx.x & (64 * NW - 1); }      // among the waves of the operand
  typedef uint8_t T;
  static constexpr bool COPIES = false;
  static constexpr int CHUNKS = R * 4 / (64 * NW);
  static constexpr int PIECES = CHUNKS;
  static_assert(R * 4 % (64 * NW) == 0, "whole chunks");
  uint4 q[CHUNKS];
  int byte[CHUNKS];
  __amdgpu_buffer_rsrc_t codes, scales;
  unsigned off[CHUNKS], scale_off[CHUNKS];
  CodeWalk walk;

  __device__ __forceinline__ void prepare(const T* base, const uint8_t* scale, long long stride, int row0, int rows, int k0, int k_end, int) {
    const long long blocks = stride / BLOCK8;
    codes = buffer_of(base + row0 * stride, (unsigned long long)(rows * stride));
    scales = buffer_of(scale + row0 * blocks, (unsigned long long)(rows * blocks));
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const int r = thread() / 4 + p * (16 * NW);
      off[p] = r < rows ? (unsigned)(r * stride) + thread() % 4 * 16 : NO_ROW;
      scale_off[p] = r < rows ? (unsigned)(r * blocks) : NO_ROW;
    }
    walk.start(k0);
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) ask(p);
    walk.started(k_end);
  }
  __device__ __forceinline__ void ask(int p) {
    // (the scalar part of an offset is outside the buffer's bounds check: walk.k itself stays in the row)
    q[p] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)off[p], walk.k, 0));
    byte[p] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)scale_off[p], walk.k / BLOCK8, 0);
  }
  __device__ __forceinline__ void next_step() {}
  __device__ __forceinline__ void piece(int p, int, int left, unsigned char* lds, unsigned) {
    const int r = thread() / 4 + p * (16 * NW), c = thread() % 4 * 2;
    const float f = power_of_two(byte[p]);
    const unsigned w[4] = {q[p].x, q[p].y, q[p].z, q[p].w};
    u32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lo[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], f, false));
      lo[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], f, true));
      hi[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], f, false));
      hi[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], f, true));
    }
    *reinterpret_cast<u32x4*>(lds + r * 128 + ((c ^ S::swap_of(r)) * 16)) = lo;
    *reinterpret_cast<u32x4*>(lds + r * 128 + (((c + 1) ^ S::swap_of(r)) * 16)) = hi;
    ask(p);
    if (p == CHUNKS - 1) walk.asked(left);
  }
};

enum Form { ALIGNED, ANY, EIGHT_BITS };
template <Form F, bool KMAJOR, int R, int NW> struct Operand { typedef Copied<KMAJOR, R, NW> type; };
template <bool KMAJOR, int R, int NW> struct Operand<ANY, KMAJOR, R, NW> { typedef Loaded<KMAJOR, R, NW> type; };
template <int R, int NW> struct Operand<EIGHT_BITS, true, R, NW> { typedef Converted<R, NW> type; };

// One tile of expert `group` (q.groups: of none): rows m0 .. m_end - 1, columns n0 .., sum indices k_begin .. k_end - 1.
template <Form F, int KIND, int BM, int BN, int WM, int WN, int S, int SPLIT, typename C>
__device__ __forceinline__ void tile_product(const LinearArgs& q, unsigned char* lds, int group, int part, int m0, int m_end, int n0, int k_begin, int k_end) {
  constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr bool EIGHT = F == EIGHT_BITS;
  typedef typename Operand<F, KIND != WGRAD, BM, NW>::type CA;
  typedef typename Operand<F, KIND == FORWARD, BN, NW>::type CB;
  typedef typename CA::T T;
  constexpr int STAGE = CA::BYTES + CB::BYTES;                    // S of them
  // SPLIT = 2: two sets of waves take half of the sum each, with stages of their own
  const int set = SPLIT == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const int all_steps = (k_end - k_begin + STEP - 1) / STEP, steps = (all_steps + SPLIT - 1) / SPLIT;
  if (SPLIT > 1) {
    k_begin = min(k_begin + set * steps * STEP, k_end);
    k_end = min(k_begin + steps * STEP, k_end);
  }
  int left = k_end - k_begin;

  floatx4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (steps > 0) {
    const int expert = KIND == WGRAD ? 0 : group;
    CA ca;
    CB cb;
    const long long blocks8 = (long long)q.n * (q.b_stride / BLOCK8);
    ca.prepare((const T*)q.a, q.a_scale, q.a_stride, m0, min(BM, m_end - m0), k_begin, k_end, wave);
    cb.prepare((const T*)q.b + expert * q.b_group, EIGHT ? q.b_scale + expert * blocks8 : nullptr, q.b_stride, n0, min(BN, q.n - n0), k_begin, k_end, wave);
    unsigned char* const whole_lds = lds;
    if (SPLIT > 1) lds += set * S * STAGE;
    const unsigned lds0 = lds_address(lds);
    constexpr int PIECES = CA::PIECES + CB::PIECES;
    auto copy_piece = [&](int p, int stage) {
      if (p < CA::PIECES) ca.piece(p, wave, left, lds + stage * STAGE, lds0 + stage * STAGE);
      else cb.piece(p - CA::PIECES, wave, left, lds + stage * STAGE + CA::BYTES, lds0 + stage * STAGE + CA::BYTES);
    };

    // Half a step is multiplied while the operands of the next half are read from LDS, so that the matrix pipe sees no wait: the second half's during the
    // first, and during the second those of the next step, whose copies have then had S - 1 steps to arrive.  The barrier between the halves
    // says that they have, and that no wave reads this step's stage any more, which the copies of step s + S overwrite.
    struct Operands { u32x4 a[TM], b[TN]; };
    Operands f0, f1;
    auto read_piece = [&](Operands& f, int p, int stage, int h) {
      const unsigned char* at = lds + stage * STAGE;
      if (p < TN) f.b[p] = CB::read(at + CA::BYTES, wn + p * 16, h);
      else f.a[p - TN] = CA::read(at, wm + (p - TN) * 16, h);
    };
    constexpr int SLOTS = TM > 2 ? TM - 1 : TM;                   // rows of products that reads and copies are issued between
    // products of `f`; meanwhile the operands `next` of half h of `stage`, and (copy) the copies of another step into `into`
    auto half_step = [&](const Operands& f, Operands& next, int stage, int h, auto copy, int into) {
      static_for<0, TM>([&](auto iv) {
        constexpr int i = iv.value;
        static_for<i * (TM + TN) / SLOTS, (i + 1) * (TM + TN) / SLOTS>([&](auto p) { if constexpr (p.value < TM + TN) read_piece(next, p.value, stage, h); });
        if constexpr (copy.value)
          static_for<i * PIECES / SLOTS, (i + 1) * PIECES / SLOTS>([&](auto p) { if constexpr (p.value < PIECES) copy_piece(p.value, into); });
#pragma unroll
        for (int j = 0; j < TN; ++j) mma(acc[i][j], f.b[j], f.a[i]);
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    // (Copies behind the last step ask for nothing and fill the stage with zeros; its operands are read and not multiplied.)
    static_assert(CA::COPIES || S == 2, "operands that go through registers are a step ahead");
#pragma unroll
    for (int s = 0; s < S; ++s) {
      ca.next_step();
      cb.next_step();
#pragma unroll
      for (int p = 0; p < PIECES; ++p) copy_piece(p, s);
      left -= STEP;
    }
    if constexpr (CA::COPIES) wait_vm<(S - 1) * PIECES>();
    __syncthreads();
    static_for<0, TM + TN>([&](auto p) { read_piece(f0, p.value, 0, 0); });
    for (int s = 0, stage = 0; s < steps; ++s) {
      const int next = stage + 1 < S ? stage + 1 : 0;
      half_step(f0, f1, stage, 1, std::false_type(), 0);
      if constexpr (CA::COPIES) wait_vm<(S - 2) * PIECES>();
      __syncthreads();
      ca.next_step();
      cb.next_step();
      half_step(f1, f0, next, 0, std::true_type(), stage);
      left -= STEP;
      stage = next;
    }
    if constexpr (CA::COPIES) wait_vm<0>();
    __syncthreads();                                              // nothing is written to LDS any more, or read
    lds = whole_lds;
  }

  if constexpr (SPLIT > 1) {                                      // the second set's sums are added to the first's
    floatx4* at = reinterpret_cast<floatx4*>(lds) + wave * 64 + (threadIdx.x & 63);
    static_assert(SPLIT == 2 && TM * TN * NW * 1024 <= 2 * S * STAGE, "the sums' LDS");
    if (set == 1)
#pragma unroll
      for (int i = 0; i < TM * TN; ++i) at[i * NW * 64] = acc[i / TN][i % TN];
    __syncthreads();
    if (set == 0)
#pragma unroll
      for (int i = 0; i < TM * TN; ++i) acc[i / TN][i % TN] += at[i * NW * 64];
    __syncthreads();
    if (set == 1) return;
  }
  C* c = (C*)q.c + (KIND == WGRAD ? part * q.part + (long long)group * q.c_group : 0);
  static_assert(NW * 16 * (TN * 16 * (int)sizeof(C) + 16) <= S * STAGE, "the outputs' LDS");
  store_rows<C, KIND == WGRAD, TM, TN>(acc, c, q.c_stride, lds + wave * 16 * (TN * 16 * (int)sizeof(C) + 16), m0 + wm, m_end, n0 + wn, q.n);
}

// Stages of a tile in a share of LDS
constexpr int stages(Form f, int height, int width, int kib) {
  const int most = kib * 1024 / ((height + width) * 128);
  return f != ALIGNED || most < 2 ? 2 : most > 4 ? 4 : most;
}
// How a launch with tiles of BM x BN by WM x WN waves (SPLIT = 2: and as many again) takes experts' last rows: in half and a quarter of the height.  Next to many
// 256 x 256 tiles, which have a CU for themselves, half the columns by two sets of four waves, twice the blocks of half the length, end a launch sooner (eight experts of
// 2048 rows, 4096 -> 4096: 489 -> 478 us, in 8 bits 486 -> 456, measured in turn); where they are most of the launch, they read the weights less well (32 of 128, 2048 -> 2048: 79 -> 92).
template <Form F, int BM, int BN, int WM, int WN, int SPLIT>
struct Shapes {
  static constexpr bool NARROW = BM == 256;
  static constexpr int KIB = NARROW ? 160 : 80, S = stages(F, BM, BN, KIB);
  static constexpr int S_HALF = stages(F, BM / 2, BN, KIB), S_QUARTER = stages(F, BM / 4, BN, KIB);
  static constexpr int S_NARROW_HALF = stages(F, BM / 2, BN / 2, KIB / 2), S_NARROW_QUARTER = stages(F, BM / 4, BN / 2, KIB / 2);
  static constexpr bool QUARTERS = F != EIGHT_BITS;               // (8-bit codes are loaded for a row by four lanes: eight waves have 128 rows at least)
  static constexpr int bytes(int height, int width, int s, int sets) { return (height + width) * 128 * s * sets; }
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int WIDE_LDS = most(bytes(BM, BN, S, SPLIT), most(bytes(BM / 2, BN, S_HALF, SPLIT), bytes(BM / 4, BN, S_QUARTER, SPLIT)));
  static constexpr int LDS = NARROW ? most(WIDE_LDS, most(bytes(BM / 2, BN / 2, S_NARROW_HALF, 2), bytes(BM / 4, BN / 2, S_NARROW_QUARTER, 2))) : WIDE_LDS;
  static_assert(LDS <= 160 * 1024, "LDS");
};

// Rows of tiles in bands of 8, columns by 4 within a band: 32 tiles in a row, which the CUs of one XCD work on together, then read 8 + 4
// panels through its L2 in place of 64.
__device__ __forceinline__ void banded(unsigned id, unsigned row_tiles, unsigned col_tiles, unsigned& r, unsigned& c) {
  const unsigned band = id / (8 * col_tiles), first = band * 8, high = min(8u, row_tiles - first), in_band = id - first * col_tiles;
  const unsigned four = in_band / (high * 4), in_four = in_band - four * (high * 4);
  r = first + in_four % high;
  c = four * 4 + in_four / high;
}

// Forward and dgrad.  Block b runs on XCD b % 8.  Each XCD takes one stretch of the tiles of full height (the whole ones, then experts' last ones of more than half
// of it), then its share of the last ones that half the height is enough for, then of those for a quarter, so that the shortest blocks end the launch.
template <Form F, int KIND, int BM, int BN, int WM, int WN, int SPLIT, typename C>
__global__ __launch_bounds__(64 * WM * WN * SPLIT, 2) void linear_kernel(LinearArgs q) {
  extern __shared__ __align__(1024) unsigned char lds[];
  typedef Shapes<F, BM, BN, WM, WN, SPLIT> P;
  unsigned count[SORTS];
  count_tiles(q.offs, q.groups, q.rows, BM, count);
  const bool narrow = P::NARROW && 4 * (count[HALF] + count[LOW]) <= count[WHOLE] + count[HIGH];
  const unsigned cols = (unsigned)(q.n + BN - 1) / BN, end_cols = narrow ? (unsigned)(q.n + BN / 2 - 1) / (BN / 2) : cols, block = block_of(q), xcd = block & 7, i = block >> 3;
  const unsigned full = (count[WHOLE] + count[HIGH]) * cols, share = (full + 7) / 8;
  unsigned r, c, id = i < share ? xcd * share + i : (i - share) * 8 + xcd;
  int sort;
  if (i < share) {
    if (id >= full) return;
    sort = id < count[WHOLE] * cols ? WHOLE : HIGH;
    if (sort == HIGH) id -= count[WHOLE] * cols;
  } else {
    sort = id < count[HALF] * end_cols ? HALF : LOW;
    if (sort == LOW) id -= count[HALF] * end_cols;
    if (id >= count[sort] * end_cols) return;
  }
  if (sort == WHOLE) {
    banded(id, count[WHOLE], cols, r, c);
  } else {
    r = id / (sort == HIGH ? cols : end_cols);
    c = id % (sort == HIGH ? cols : end_cols);
  }
  int group, m0, m_end;
  find_tile_of(sort, q.offs, q.groups, q.rows, BM, r, group, m0, m_end);
  const int k = group < q.groups ? q.k : 0;
  if (sort == WHOLE) m_end = min(m_end, m0 + BM);
  if (sort <= HIGH)
    tile_product<F, KIND, BM, BN, WM, WN, P::S, SPLIT, C>(q, lds, group, 0, m0, m_end, (int)c * BN, 0, k);
  else if (narrow) {
    if constexpr (P::NARROW) {
      if (sort == HALF) tile_product<F, KIND, BM / 2, BN / 2, WM, WN / 2, P::S_NARROW_HALF, 2, C>(q, lds, group, 0, m0, m_end, (int)c * (BN / 2), 0, k);
      else tile_product<F, KIND, BM / 4, BN / 2, WM, WN / 2, P::S_NARROW_QUARTER, 2, C>(q, lds, group, 0, m0, m_end, (int)c * (BN / 2), 0, k);
    }
  } else if (!P::QUARTERS || sort == HALF) {
    tile_product<F, KIND, BM / 2, BN, WM, WN, P::S_HALF, SPLIT, C>(q, lds, group, 0, m0, m_end, (int)c * BN, 0, k);
  } else if constexpr (P::QUARTERS) {
    tile_product<F, KIND, BM / 4, BN, WM, WN, P::S_QUARTER, SPLIT, C>(q, lds, group, 0, m0, m_end, (int)c * BN, 0, k);
  }
}

template <Form F, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void linear_wgrad_kernel(LinearArgs q) {
  extern __shared__ __align__(1024) unsigned char lds[];
  const unsigned block = block_of(q);
  const int n_tiles = (q.n + BN - 1) / BN, m_tiles = (q.m + BM - 1) / BM, t = block / n_tiles, e = t / m_tiles, group = e / q.parts, part = e % q.parts;
  int begin, end;
  group_rows(q.offs, q.groups, q.rows, group, begin, end);
  part_of(part, q.parts, begin, end);
  tile_product<F, WGRAD, BM, BN, WM, WN, Shapes<F, BM, BN, WM, WN, 1>::S, 1, float>(q, lds, group, part, t % m_tiles * BM, q.m, (int)(block % n_tiles) * BN, begin, end);
}

// dw = the parts, added in order
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* parts, float* dw, long long n, int count) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    float s = parts[i];
    for (int p = 1; p < count; ++p) s += parts[p * n + i];
    dw[i] = s;
  }
}

// ---- few rows ----
//
// Tiles of 16 TM rows and few columns, whose sum the block's waves share: wave w takes the chunks w, w + NW, ... of it, straight from memory into MFMA
// operands, and the waves' sums are joined in order through LDS.  Bound by the weights' bytes: every lane has U loads of 16 bytes of them in flight and more of the rows.
// A lane's 16 bytes of a k-major operand are one row's; of dgrad's weights, whose sum index is the row, they are neighbouring columns of one
// row: column 8 c + j (bf16; 4 c + j in fp32) of the tile is column c = l % 16 of MFMA j.  fp32 goes through the fp32 MFMA.
template <typename T> struct Few;                                 // EACH: elements of 16 bytes; DEEP: sum indices that four lanes' 16 bytes of a row cover
template <> struct Few<float> { static constexpr int EACH = 4, DEEP = 16; };
template <> struct Few<bf16_t> { static constexpr int EACH = 8, DEEP = 32; };
template <> struct Few<uint8_t> { static constexpr int EACH = 16, DEEP = 64; };

__device__ __forceinline__ u32x4 load16(const __amdgpu_buffer_rsrc_t& b, unsigned off) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)off, 0, 0)); }

// the first `left` of four fp32 values
__device__ __forceinline__ u32x4 first_of(u32x4 v, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < left ? v[i] : 0u;
  return v;
}

struct Pair8 { u32x4 lo, hi; };
__device__ __forceinline__ Pair8 to_bf16(const u32x4& q, int byte) {
  const float f = power_of_two(byte);
  Pair8 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    r.lo[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], f, false));
    r.lo[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], f, true));
    r.hi[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[2 + i], f, false));
    r.hi[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[2 + i], f, true));
  }
  return r;
}

// Sums of the waves for each lane's Q quads of outputs, added in the waves' order; eight quads at a time.
template <int Q, int NW, typename F>
__device__ __forceinline__ void join_waves(const floatx4 (&acc)[Q], F&& write) {
  constexpr int EIGHT = Q < 8 ? Q : 8;
  static_assert(Q % EIGHT == 0, "whole eights");
  __shared__ float4 part[NW][EIGHT][64];
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
#pragma unroll
  for (int first = 0; first < Q; first += EIGHT) {
    if (first) __syncthreads();
#pragma unroll
    for (int k = 0; k < EIGHT; ++k) part[wave][k][l] = make_float4(acc[first + k][0], acc[first + k][1], acc[first + k][2], acc[first + k][3]);
    __syncthreads();
    for (int k = wave; k < EIGHT; k += NW) {
      float4 v = part[0][k][l];
#pragma unroll
      for (int w = 1; w < NW; ++w) {
        const float4 o = part[w][k][l];
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      }
      const float f[4] = {v.x, v.y, v.z, v.w};
      write(first + k, f);
    }
  }
}

// Forward: JT sixteens of columns; U chunks of DEEP sum indices a turn.
template <typename T, int TM, int JT, int U, int NW, bool ANY_ROWS, typename C>
__global__ __launch_bounds__(64 * NW) void linear_few_kernel(LinearArgs q) {
  constexpr int EACH = Few<T>::EACH, DEEP = Few<T>::DEEP, ES = (int)sizeof(T);
  const int cols = (q.n + 16 * JT - 1) / (16 * JT);
  const unsigned block = block_of(q);
  const int column = (int)(block % cols), n0 = column * 16 * JT;
  int group, m0, m_end;
  if (!find_tile(q.offs, q.groups, q.rows, 16 * TM, block / cols, group, m0, m_end)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  floatx4 acc[TM * JT];
#pragma unroll
  for (int i = 0; i < TM * JT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (group < q.groups) {
    const int rows = min(16 * TM, m_end - m0), outs = min(16 * JT, q.n - n0);
    const T *x_rows = (const T*)q.a + m0 * q.a_stride, *w_rows = (const T*)q.b + group * q.b_group + n0 * q.b_stride;
    const __amdgpu_buffer_rsrc_t x = buffer_of(x_rows, (unsigned long long)(((rows - 1) * q.a_stride + q.k) * ES));
    const __amdgpu_buffer_rsrc_t w = buffer_of(w_rows, (unsigned long long)(((outs - 1) * q.b_stride + q.k) * ES));
    const long long blocks = q.b_stride / BLOCK8;
    const __amdgpu_buffer_rsrc_t xs = buffer_of(q.a_scale + m0 * blocks, (unsigned long long)(rows * blocks));
    const __amdgpu_buffer_rsrc_t ws = buffer_of(q.b_scale + (group * (long long)q.n + n0) * blocks, (unsigned long long)(outs * blocks));
    unsigned xo[TM], wo[JT];                                      // (rows that are none lie behind the buffers' ends)
#pragma unroll
    for (int i = 0; i < TM; ++i) xo[i] = (unsigned)((i * 16 + (l & 15)) * q.a_stride * ES);
#pragma unroll
    for (int j = 0; j < JT; ++j) wo[j] = (unsigned)((j * 16 + (l & 15)) * q.b_stride * ES);
    // Neighbouring tiles of columns start at different places of the sum: with rows of 8 KiB all of them would ask the same few memory channels at a time.
    const int turns = (q.k + NW * DEEP * U - 1) / (NW * DEEP * U), start = column % turns;
    for (int turn = 0; turn < turns; ++turn) {
      const int k0 = ((turn + start < turns ? turn + start : turn + start - turns) * NW + wave) * DEEP * U;
      u32x4 fx[U][TM], fw[U][JT];
      int bx[U][TM], bw[U][JT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + u * DEEP + (l >> 4) * EACH;
        const bool in = k < q.k;
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          if constexpr (ANY_ROWS) fw[u][j] = load_last(w_rows + (long long)(j * 16 + (l & 15)) * q.b_stride + k, j * 16 + (l & 15) < outs ? q.k - k : 0, q.k < 8);
          else fw[u][j] = load16(w, in ? wo[j] + k * ES : NO_ROW);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if constexpr (ANY_ROWS) fx[u][i] = load_last(x_rows + (long long)(i * 16 + (l & 15)) * q.a_stride + k, i * 16 + (l & 15) < rows ? q.k - k : 0, q.k < 8);
          else fx[u][i] = load16(x, in ? xo[i] + k * ES : NO_ROW);
        }
        if constexpr (ES == 1) {
#pragma unroll
          for (int j = 0; j < JT; ++j) bw[u][j] = __builtin_amdgcn_raw_buffer_load_b8(ws, in ? (j * 16 + (l & 15)) * (int)blocks + k / BLOCK8 : (int)NO_ROW, 0, 0);
#pragma unroll
          for (int i = 0; i < TM; ++i) bx[u][i] = __builtin_amdgcn_raw_buffer_load_b8(xs, in ? (i * 16 + (l & 15)) * (int)blocks + k / BLOCK8 : (int)NO_ROW, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);                          // (all of them in flight before the first is waited for)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (ES == 4) {
          const int left = q.k - (k0 + u * DEEP + (l >> 4) * EACH);
          if (q.k % EACH) {                                       // (the values behind a row's last are the next row's)
#pragma unroll
            for (int j = 0; j < JT; ++j) fw[u][j] = first_of(fw[u][j], left);
#pragma unroll
            for (int i = 0; i < TM; ++i) fx[u][i] = first_of(fx[u][i], left);
          }
        }
        if constexpr (ANY_ROWS) {
          const int left = q.k - (k0 + u * DEEP + (l >> 4) * EACH);
#pragma unroll
          for (int j = 0; j < JT; ++j) fw[u][j] = shift_last(fw[u][j], left, q.k < 8);
#pragma unroll
          for (int i = 0; i < TM; ++i) fx[u][i] = shift_last(fx[u][i], left, q.k < 8);
        }
        Pair8 px[TM];
        if constexpr (ES == 1)
#pragma unroll
          for (int i = 0; i < TM; ++i) px[i] = to_bf16(fx[u][i], bx[u][i]);
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          if constexpr (ES == 1) {
            const Pair8 pw = to_bf16(fw[u][j], bw[u][j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
              mma(acc[i * JT + j], pw.lo, px[i].lo);
              mma(acc[i * JT + j], pw.hi, px[i].hi);
            }
          } else {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
              if constexpr (ES == 2) {
                mma(acc[i * JT + j], fw[u][j], fx[u][i]);
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  acc[i * JT + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(fw[u][j][e]), __uint_as_float(fx[u][i][e]), acc[i * JT + j], 0, 0, 0);
              }
            }
          }
        }
      }
    }
  }
  join_waves<TM * JT, NW>(acc, [&](int k, const float (&v)[4]) {
    const int m = m0 + k / JT * 16 + (l & 15), n = n0 + k % JT * 16 + (l >> 4) * 4;
    if (m < m_end && n < q.n) store_four<C>((C*)q.c + (long long)m * q.c_stride + n, q.n - n, v);
  });
}

// dgrad: sixteen lanes' 16 bytes of columns; 8 (bf16) or 4 (fp32) sum indices for each load of the rows.
template <typename T, int TM, int U, int NW, bool ANY_ROWS>
__global__ __launch_bounds__(64 * NW) void linear_few_dgrad_kernel(LinearArgs q) {
  constexpr int EACH = Few<T>::EACH, DEEP = Few<T>::DEEP, ES = (int)sizeof(T), BN = 16 * EACH;
  const int cols = (q.n + BN - 1) / BN;
  const unsigned block = block_of(q);
  const int n0 = (int)(block % cols) * BN;
  int group, m0, m_end;
  if (!find_tile(q.offs, q.groups, q.rows, 16 * TM, block / cols, group, m0, m_end)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  floatx4 acc[TM * EACH];
#pragma unroll
  for (int i = 0; i < TM * EACH; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (group < q.groups) {
    const int rows = min(16 * TM, m_end - m0), col = n0 + (l & 15) * EACH;
    const T *x_rows = (const T*)q.a + m0 * q.a_stride, *w_rows = (const T*)q.b + group * q.b_group;
    const __amdgpu_buffer_rsrc_t x = buffer_of(x_rows, (unsigned long long)(((rows - 1) * q.a_stride + q.k) * ES));
    const __amdgpu_buffer_rsrc_t w = buffer_of(w_rows, (unsigned long long)(((q.k - 1) * q.b_stride + q.n) * ES));
    unsigned xo[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) xo[i] = (unsigned)((i * 16 + (l & 15)) * q.a_stride * ES);
    for (int k0 = wave * DEEP * U; k0 < q.k; k0 += NW * DEEP * U) {
      u32x4 fx[U][TM], fw[U][EACH];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + u * DEEP + (l >> 4) * EACH;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          if constexpr (ANY_ROWS) fw[u][e] = load_last(w_rows + (k + e) * q.b_stride + col, k + e < q.k ? q.n - col : 0, q.n < 8);
          else fw[u][e] = load16(w, k + e < q.k && col < q.n ? (unsigned)(((k + e) * q.b_stride + col) * ES) : NO_ROW);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if constexpr (ANY_ROWS) fx[u][i] = load_last(x_rows + (long long)(i * 16 + (l & 15)) * q.a_stride + k, i * 16 + (l & 15) < rows ? q.k - k : 0, q.k < 8);
          else fx[u][i] = load16(x, k < q.k ? xo[i] + k * ES : NO_ROW);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (ANY_ROWS) {
#pragma unroll
          for (int e = 0; e < EACH; ++e) fw[u][e] = shift_last(fw[u][e], q.n - col, q.n < 8);
#pragma unroll
          for (int i = 0; i < TM; ++i) fx[u][i] = shift_last(fx[u][i], q.k - (k0 + u * DEEP + (l >> 4) * EACH), q.k < 8);
        }
        if constexpr (ES == 4) {
          if (q.k % EACH)
#pragma unroll
            for (int i = 0; i < TM; ++i) fx[u][i] = first_of(fx[u][i], q.k - (k0 + u * DEEP + (l >> 4) * EACH));
#pragma unroll
          for (int j = 0; j < EACH; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
              for (int e = 0; e < EACH; ++e)
                acc[i * EACH + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(fx[u][i][e]), __uint_as_float(fw[u][e][j]), acc[i * EACH + j], 0, 0, 0);
        } else {
#pragma unroll
          for (int j = 0; j < EACH; ++j) {                          // column j of the lane's: element j of its eight loads
            u32x4 b;
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = __builtin_amdgcn_perm(fw[u][2 * e + 1][j / 2], fw[u][2 * e][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int i = 0; i < TM; ++i) mma(acc[i * EACH + j], fx[u][i], b);
          }
        }
      }
    }
  }
  // acc[i][j][e]: row 16 i + 4 (l / 16) + e, column EACH (l % 16) + j; neighbouring columns together
  floatx4 out[TM * EACH];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < EACH / 4; ++h)
        out[(i * 4 + e) * (EACH / 4) + h] = floatx4{acc[i * EACH + 4 * h][e], acc[i * EACH + 4 * h + 1][e], acc[i * EACH + 4 * h + 2][e], acc[i * EACH + 4 * h + 3][e]};
  join_waves<TM * EACH, NW>(out, [&](int k, const float (&v)[4]) {
    const int h = k % (EACH / 4), e = k / (EACH / 4) % 4, m = m0 + k / EACH * 16 + (l >> 4) * 4 + e, n = n0 + (l & 15) * EACH + 4 * h;
    if (m < m_end && n < q.n) store_four<T>((T*)q.c + (long long)m * q.c_stride + n, q.n - n, v);
  });
}

// ---- launches ----

constexpr long long MOST_BLOCKS = 0x7fffffff;

// A launch has fewer than 2^32 threads (the runtime takes more of them modulo 2^32, without an error): blocks beyond go to another, in eights, which keep their XCDs.
gan_status launch(void (*kernel)(LinearArgs), long long blocks, int threads, int lds, LinearArgs q, hipStream_t st) {
  if (blocks > MOST_BLOCKS) return operator_fail(GAN_E_SHAPE, "more than 2^31 - 1 tiles");
  if (lds > 65536 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) {
    (void)hipGetLastError();
    return operator_fail(GAN_E_HIP, "the kernel's LDS could not be set");
  }
  const long long most = (1ll << 31) / threads;
  operator_launches();
  for (long long first = 0; first < blocks; first += most) {
    q.first = (unsigned)first;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(most, blocks - first)), dim3(threads), lds, st, q);
  }
  return operator_launched();
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
// experts that have rows, at most
long long most_groups(const LinearArgs& q) { return std::max(1, std::min(q.groups, q.rows)); }
long long tiles(const LinearArgs& q, int height, int width) { return (q.rows / height + most_groups(q)) * ceil_div(q.n, width); }
long long wgrad_tiles(long long groups, long long m, long long n, int side) { return groups * ceil_div(m, side) * ceil_div(n, side); }

template <Form F, int KIND, int BM, int BN, int WM, int WN, int SPLIT, typename C>
gan_status launch_tiles(const LinearArgs& q, hipStream_t st) {
  typedef Shapes<F, BM, BN, WM, WN, SPLIT> P;
  if constexpr (KIND == WGRAD) {
    return launch(linear_wgrad_kernel<F, BM, BN, WM, WN>, q.parts * wgrad_tiles(q.groups, q.m, q.n, BM), 64 * WM * WN, P::bytes(BM, BN, P::S, 1), q, st);
  } else {
    // Full tiles and lower ones are each shared among the eight XCDs; narrow ones are twice as many, but then a fifth of the tiles at most.
    const long long high = most_tiles(q.rows, q.groups, BM), blocks = (high + (P::NARROW ? ceil_div(high, 5) : 0)) * ceil_div(q.n, BN);
    return launch(linear_kernel<F, KIND, BM, BN, WM, WN, SPLIT, C>, 8 * (ceil_div(blocks, 8) + 1), 64 * WM * WN * SPLIT, P::LDS, q, st);
  }
}

// 256 x 256 tiles where they fill the CUs and experts have more than 32 rows on average, 128 x 128 where not.  Both sides, us on an MI355X from cold memory (256, 128):
// 32 experts of 128 rows, 2048 -> 2048, forward 77, 97; 64 of 47, 1024 -> 1024, dgrad 31, 34; 128 of 14, 2361 -> 384, 8 bits 59, 43; four of 175, 4096 -> 4096 (64 tiles
// of 256), forward 100, 67; weight gradient of 64 experts, 2816 -> 512: 109, 138 (through the caches).  Where those leave about one block to a CU and the sum is long, two sets of waves take half of
// it each (without, with): one expert of 1000 rows, 4096 -> 4096: 62, 53, in 8 bits 60, 43; one of 600, 1024 -> 1024: 16.9, 14.2; ten of 128, 512 -> 1024 (8 steps): 11.7, 11.8.
template <Form F, int KIND, typename C>
gan_status launch_large(const LinearArgs& q, hipStream_t st) {
  const bool big = KIND == WGRAD ? q.parts * wgrad_tiles(q.groups, q.m, q.n, 256) >= 256 : tiles(q, 256, 256) >= 256 && q.rows / most_groups(q) > 32;
  if constexpr (F != ANY)
    if (big) return launch_tiles<F, KIND, 256, 256, 2, 4, 1, C>(q, st);
  if constexpr (KIND != WGRAD)
    if (tiles(q, 128, 128) <= 288 && q.k >= 512) return launch_tiles<F, KIND, 128, 128, 2, 2, 2, C>(q, st);
  return launch_tiles<F, KIND, 128, 128, 2, 2, 1, C>(q, st);
}

// blocks of 32 columns, at most
long long few_blocks(const LinearArgs& q) { return most_groups(q) * ceil_div(q.n, 32); }
template <typename T, int TM, int JT, int U, bool ANY_ROWS, typename C>
gan_status launch_few_as(const LinearArgs& q, hipStream_t st) {
  return launch(linear_few_kernel<T, TM, JT, U, 8, ANY_ROWS, C>, most_tiles(q.rows, q.groups, 16 * TM) * ceil_div(q.n, 16 * JT), 512, 0, q, st);
}
template <typename T, bool ANY_ROWS, typename C>
gan_status launch_few(const LinearArgs& q, int sixteens, hipStream_t st) {
  constexpr int U = sizeof(T) == 1 ? 2 : 4;
  if (sixteens == 2) return launch_few_as<T, 2, 2, U, ANY_ROWS, C>(q, st);
  // sixteen columns a block where 32 make few blocks: eight rows of eight experts, 4096 -> 4096, 28 us (32 columns: 35); four rows of a hundred, 1024 -> 1024, 47 (36).  A turn
  // of the eight waves takes in 1024 sum indices of bf16, or half of that where there are fewer than two such (ten rows of a hundred experts, 1024 -> 1024: 9.2 -> 7.9;
  // but eight of eight, 4096 -> 4096: 31 -> 39)
  if (few_blocks(q) <= 1024) return q.k < 2048 ? launch_few_as<T, 1, 1, 2, ANY_ROWS, C>(q, st) : launch_few_as<T, 1, 1, U, ANY_ROWS, C>(q, st);
  return launch_few_as<T, 1, 2, 2, ANY_ROWS, C>(q, st);
}
template <typename T, int TM, int U, int NW, bool ANY_ROWS>
gan_status launch_few_dgrad_as(const LinearArgs& q, hipStream_t st) {
  return launch(linear_few_dgrad_kernel<T, TM, U, NW, ANY_ROWS>, most_tiles(q.rows, q.groups, 16 * TM) * ceil_div(q.n, 16 * Few<T>::EACH), 64 * NW, 0, q, st);
}
template <typename T, bool ANY_ROWS>
gan_status launch_few_dgrad(const LinearArgs& q, int sixteens, hipStream_t st) {
  if constexpr (sizeof(T) == 4) return launch_few_dgrad_as<T, 1, 2, 8, false>(q, st);
  else return sixteens == 2 ? launch_few_dgrad_as<T, 2, 2, 8, ANY_ROWS>(q, st) : launch_few_dgrad_as<T, 1, 2, 8, ANY_ROWS>(q, st);
}

// Sixteens of rows for the kernel for few rows, or 0 where tiles are faster: up to 8 rows an expert, whose weights then are the time (a hundred experts of 4 rows,
// 1024 -> 1024, forward: 43 us, 45 in 128 x 128 tiles; one row of one, 4096 -> 4096: 7.5, 37), and where there are few outputs (one expert of 200 rows, 4096 -> 1024: 18 us, 49;
// four of 175, 4096 -> 4096: 171, 66).
// In fp32 (us by this kernel, in tiles) up to 24 rows an expert forward (16 experts of 25, 2048 -> 2048: 76, 93; a hundred of 24, 1024 -> 1024: 122, 122; 32 of 29,
// 640 -> 2176: 82, 62) and up to 32 in dgrad (a hundred of 24: 107, 121; 32 of 29, 640 <- 2176: 69, 91).  Beyond, where 64 x 64 tiles are few, forward: four of 100, 2048 -> 2048
// (320 tiles): 64, 73; 32 of 25, 512 -> 512 (352): 16, 19.5; four of 175, 2048 -> 2048 (480): 94, 81; two of 1000, 1024 -> 1024 (530): 62, 44.  And where 128 x 128 tiles
// are few in dgrad, whose columns this kernel reads more widely: ten of 111, 110 <- 6272: 47, 222; eight of 244, 1024 <- 2808 (184): 132, 153; ten of 640, 784 <- 512 (420): 71, 53.
// This rule and the tiles' see the average number of rows, which the host knows, not the offsets: a batch that is all one expert's is taken like one of average experts (800 rows of
// one of a hundred, 1024 -> 1024, bf16: 27 us forward, 15 dgrad; the same rows with that expert alone 14, 14; fp32 43, 25 and 34, 26).
int few_rows(const LinearArgs& q, int kind, int esize) {
  const long long each = q.rows / most_groups(q);
  // short sums of many outputs give the waves little to share (128 experts of 3.5 rows, 256 -> 896: 32 us, 21 in tiles; fp32, eight of 128, 64 -> 896: 15.3, 5.6)
  if (q.k < 512 && (few_blocks(q) > 1024 || (esize == 4 && each > 8))) return 0;
  if (each <= 8) return 1;
  if (esize == 4 && kind == DGRAD) return each <= 32 || tiles(q, 128, 128) < 256 ? 1 : 0;
  // (twelve rows each of a hundred, 1024 -> 1024: 103 us by sixteens, 113 by 32; twenty: 104, 87)
  if (esize == 4) return each <= 12 ? 1 : each <= 24 || tiles(q, 64, 64) <= 384 ? 2 : 0;
  return (long long)q.rows * q.n <= 1 << 19 ? 2 : 0;
}

template <int RT>
gan_status launch_fp32_as(int kind, const LinearArgs& q, hipStream_t st) {
  const long long blocks = kind == WGRAD ? q.parts * wgrad_tiles(q.groups, q.m, q.n, RT) : ceil_div(q.n, RT) * most_tiles(q.rows, q.groups, RT);
  return launch(kind == FORWARD ? linear_fp32_kernel<FORWARD, RT> : kind == DGRAD ? linear_fp32_kernel<DGRAD, RT> : linear_fp32_kernel<WGRAD, RT>, blocks, 256, 0, q, st);
}
// 128 x 128 tiles from 1024 of them on, four to a CU, in the weight gradient from 400; else 64 x 64.  us by 64, by 128.  Forward: four experts of 750 rows, 640 -> 640 (135 tiles of 128) 28, 45; 16 of
// 128, 1024 -> 1024 (256) 52, 72; eight of 512, 2048 -> 2048 (640, an expert's last one mostly empty) 272, 288; ten of 112, 110 -> 6272 (882) 29, 33; one of 8192, 2048 -> 2048 (1040) 472, 370; 32 of 200,
// 512 -> 2048 (1312) 130, 102; one of 16384, 1024 -> 4096 (4128) 922, 736.  It loses where fewer tiles are all whole (one of 4096, 2048 -> 2048, 528: 249, 199) and where more are not (a hundred of 64,
// 1024 -> 1024, 1200: 169, 178).  Weight gradient: two of 512 x 784 (56) 19, 39; three of 1024 x 1024 (192) 29, 37; ten of 512 x 784 (280) 18, 20; 16 of 768 x 512 (384) 21.5, 19.8; ten of
// 6272 x 110 (490) 26.7, 26.3; eight of 1024 x 1024 (512) 134, 107; one of 512 x 512 in 32 parts (512) 85, 69; a hundred of 512 x 512 (1600) 48, 46.
gan_status launch_fp32(int kind, const LinearArgs& q, hipStream_t st) {
  const long long large = kind == WGRAD ? q.parts * wgrad_tiles(q.groups, q.m, q.n, 128) : tiles(q, 128, 128);
  return large >= (kind == WGRAD ? 400 : 1024) ? launch_fp32_as<128>(kind, q, st) : launch_fp32_as<64>(kind, q, st);
}

// Into how many parts the weight gradient takes an expert's rows: few tiles of long sums would leave most CUs idle.  As many as make two tiles of 128 a CU, of 256 rows at least, 64 at
// most.  us, in one part and so: one expert of 16384 rows, 512 x 512 (32 parts), fp32 543, 77, bf16 150, 38; 128 x 128 (64) 441, 37 and 157, 33; one of 1000, 256 x 256 (3) 31, 16.5 and
// 14.0, 11.6; four of 1000, 512 x 512 (3) 33, 26 and 15.6, 15.5; one of 4000, 2048 x 2048 (2) 248, 195, but in bf16, whose tiles of 256 are enough, 47, 57.  Half as many tiles: the first
// 90 and 31; twice as many: 96 and 54.  Parts of 128 rows: 256 x 256 13.0 and 11.6, but 512 x 512 of 1000 rows 32 and 20.6; of 512 rows: 31 and 14, 33.5 and 15.6.
int wgrad_parts(int groups, long long rows, int n_in, int n_out) {
  const long long blocks = wgrad_tiles(groups, n_out, n_in, 128), each = rows / std::max(1, groups);
  return (int)std::max(1ll, std::min({512 / std::max(1ll, blocks), each / 256, 64ll}));
}

// by_row: the two matrices that have `rows` rows; by_group: the one of `groups` matrices.  What has no elements may be NULL.
gan_status check(int32_t precision, const void* by_row0, const void* by_row1, const void* by_group, const int32_t* offs, int32_t groups, int64_t rows, int32_t n_in, int32_t n_out) {
  if (precision != GAN_FP32 && precision != GAN_BF16_FP32MASTER) return operator_fail(GAN_E_ARG, "unknown precision");
  if ((rows > 0 && (!by_row0 || !by_row1)) || (groups > 0 && !by_group) || !offs) return operator_fail(GAN_E_ARG, "an operand is NULL");
  if (groups < 0 || rows < 0 || n_in < 1 || n_out < 1) return operator_fail(GAN_E_ARG, "negative groups or rows, or no inputs or outputs");
  if (groups > 65535 || rows > 1 << 30 || n_in > 1 << 28 || n_out > 1 << 28) return operator_fail(GAN_E_SHAPE, "more than 65535 groups, 2^30 rows, or 2^28 inputs or outputs");
  return GAN_OK;
}

// whether a step's memory of one operand stays within the 32 bits of a copy's offsets: 256 rows or 64 sum indices
bool short_rows(long long stride, int esize) { return stride * esize <= (1ll << 31) / 512; }

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" gan_status gan_group_linear(int32_t precision, const void* x, int64_t x_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                       int32_t n_in, int32_t n_out, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(precision, x, y, w, offs, groups, rows, n_in, n_out)) return s;
  if (x_stride < n_in || y_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or y_stride below n_out");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs q = {x, w, nullptr, nullptr, y, offs, x_stride, n_in, y_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_out, n_in, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(x_stride, e) && short_rows(n_in, e), aligned = small && n_in % 8 == 0 && rows_aligned16(x, x_stride, e) && aligned16(w);
  const int few = few_rows(q, FORWARD, e);
  if (precision == GAN_FP32) return few && small ? launch_few<float, false, float>(q, few, st) : launch_fp32(FORWARD, q, st);
  if (few && small) return aligned ? launch_few<bf16_t, false, bf16_t>(q, few, st) : launch_few<bf16_t, true, bf16_t>(q, few, st);
  return aligned ? launch_large<ALIGNED, FORWARD, bf16_t>(q, st) : launch_large<ANY, FORWARD, bf16_t>(q, st);
}

extern "C" gan_status gan_group_linear_dgrad(int32_t precision, const void* dy, int64_t dy_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                             int32_t n_in, int32_t n_out, void* dx, int64_t dx_stride, void* hip_stream) {
  if (const gan_status s = check(precision, dy, dx, w, offs, groups, rows, n_in, n_out)) return s;
  if (dy_stride < n_out || dx_stride < n_in) return operator_fail(GAN_E_ARG, "dy_stride is below n_out, or dx_stride below n_in");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs q = {dy, w, nullptr, nullptr, dx, offs, dy_stride, n_in, dx_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_in, n_out, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(dy_stride, e) && short_rows(n_in, e), aligned = small && n_out % 8 == 0 && n_in % 8 == 0 && rows_aligned16(dy, dy_stride, e) && aligned16(w);
  const int few = small && (long long)n_in * n_out * e < 1ll << 31 ? few_rows(q, DGRAD, e) : 0;
  if (precision == GAN_FP32) return few ? launch_few_dgrad<float, false>(q, few, st) : launch_fp32(DGRAD, q, st);
  if (few) return aligned ? launch_few_dgrad<bf16_t, false>(q, few, st) : launch_few_dgrad<bf16_t, true>(q, few, st);
  return aligned ? launch_large<ALIGNED, DGRAD, bf16_t>(q, st) : launch_large<ANY, DGRAD, bf16_t>(q, st);
}

extern "C" int64_t gan_group_linear_wgrad_bytes(int32_t groups, int64_t rows, int32_t n_in, int32_t n_out) {
  if (groups < 1 || rows < 1 || n_in < 1 || n_out < 1) return 0;
  const int parts = wgrad_parts(groups, rows, n_in, n_out);
  return parts > 1 ? (int64_t)parts * groups * n_in * n_out * (int64_t)sizeof(float) : 0;
}

extern "C" gan_status gan_group_linear_wgrad(int32_t precision, const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, const int32_t* offs,
                                             int32_t groups, int64_t rows, int32_t n_in, int32_t n_out, float* dw, void* work, int64_t work_bytes, void* hip_stream) {
  if (const gan_status s = check(precision, x, dy, dw, offs, groups, rows, n_in, n_out)) return s;
  if (x_stride < n_in || dy_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or dy_stride below n_out");
  const int64_t need = gan_group_linear_wgrad_bytes(groups, rows, n_in, n_out);
  if (work_bytes < need || (need > 0 && !work) || !aligned16(work)) return operator_fail(GAN_E_ARG, "work is smaller than gan_group_linear_wgrad_bytes, or not 16-byte aligned");
  if (groups == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2, parts = rows > 0 ? wgrad_parts(groups, rows, n_in, n_out) : 1;
  const long long n = (long long)groups * n_in * n_out;
  const LinearArgs q = {dy, x, nullptr, nullptr, parts > 1 ? work : dw, offs, dy_stride, x_stride, n_in, 0, (long long)n_in * n_out, groups, (int)rows, n_out, n_in, 0, parts, n, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool aligned = short_rows(x_stride, e) && short_rows(dy_stride, e) && n_in % 8 == 0 && n_out % 8 == 0 && rows_aligned16(x, x_stride, e) && rows_aligned16(dy, dy_stride, e);
  const gan_status s = precision == GAN_FP32 ? launch_fp32(WGRAD, q, st) : aligned ? launch_large<ALIGNED, WGRAD, float>(q, st) : launch_large<ANY, WGRAD, float>(q, st);
  if (s != GAN_OK || parts == 1) return s;
  hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)std::min(ceil_div(n, 256), 4096ll)), dim3(256), 0, st, (const float*)work, dw, n, parts);
  return operator_launched();
}

extern "C" gan_status gan_group_linear8(const uint8_t* x8, const uint8_t* x_scale, const uint8_t* w8, const uint8_t* w_scale, const int32_t* offs, int32_t groups,
                                        int64_t rows, int32_t n_in, int32_t n_out, int32_t y_precision, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(y_precision, x8, y, w8, offs, groups, rows, n_in, n_out)) return s;
  if ((rows > 0 && !x_scale) || (groups > 0 && !w_scale)) return operator_fail(GAN_E_ARG, "x_scale or w_scale is NULL");
  if (!aligned16(x8) || !aligned16(w8)) return operator_fail(GAN_E_ARG, "x8 or w8 is not 16-byte aligned");
  if (y_stride < n_out) return operator_fail(GAN_E_ARG, "y_stride is below n_out");
  const long long k = padded8(n_in);
  if (!short_rows(k, 1)) return operator_fail(GAN_E_SHAPE, "more than 2^22 inputs in 8 bits");
  if (rows == 0) return GAN_OK;
  const LinearArgs q = {x8, w8, x_scale, w_scale, y, offs, k, k, y_stride, k * n_out, 0, groups, (int)rows, 0, n_out, (int)k, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (const int few = few_rows(q, FORWARD, 1))
    return y_precision == GAN_FP32 ? launch_few<uint8_t, false, float>(q, few, st) : launch_few<uint8_t, false, bf16_t>(q, few, st);
  return y_precision == GAN_FP32 ? launch_large<EIGHT_BITS, FORWARD, float>(q, st) : launch_large<EIGHT_BITS, FORWARD, bf16_t>(q, st);
}
