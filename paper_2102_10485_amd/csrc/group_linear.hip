// Matrix products grouped by label: every expert's rows times its own weights, the gradient of the rows, and that of the weights; in fp32,
// bf16 and 8 bits.
//
//   forward   y[i]  = w[g] x[i]              C(m, n) = sum_k A(m, k) B(n, k):   A = x,  B = w[g],  k = inputs
//   dgrad     dx[i] = dy[i] w[g]                                                A = dy, B = w[g]^T, k = outputs
//   wgrad     dw[g] = sum of dy[i]^T x[i]                                       A = dy^T, B = x^T, k = g's rows
//
// "k-major" below: the sum's index runs along memory (both operands of the forward product, dy of dgrad); the others have it as the row.
// Which expert a tile of rows belongs to every wave finds itself from the offsets, so that a call is one launch.
#include "group_tiles.h"
#include "lds_copy.h"
#include "operators.h"
#include "split_mfma.h"

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
  int vec;                                     // any-alignment kernel: 16-byte loads of a (bit 0), of b (bit 1), 16-byte stores (bit 2)
};

// ---- any alignment, fp32 and bf16 ----
//
// 128 x 128 tiles, 32 of the sum's index at a time: loaded into registers while the last ones are multiplied, then written to LDS as bf16, in fp32
// as three planes of parts (split_mfma.h).  What has the sum's index as its row is kept that way and read with transposing LDS reads.
constexpr int RT = 128, RK = 32;

template <typename T, bool KMAJOR>
struct Staged {
  static constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  static constexpr int PLANE = RT * RK * 2;
  float v[2][8];

  // thread t's two chunks of eight: k-major row t / 4 (+ 64), elements 8 (t % 4) ..; else sum index t / 16 (+ 16), columns 8 (t % 16) ..
  __device__ __forceinline__ void load(const T* p, long long stride, int row0, int rows, int k0, int k_end, bool vec) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = KMAJOR ? row0 + threadIdx.x / 4 + 64 * h : k0 + threadIdx.x / 16 + 16 * h;
      const int c = KMAJOR ? k0 + threadIdx.x % 4 * 8 : row0 + threadIdx.x % 16 * 8;
      const int left = r < (KMAJOR ? rows : k_end) ? (KMAJOR ? k_end : rows) - c : 0;
      const T* at = p + (long long)r * stride + c;
      if (vec) load8<T, true>(at, left, v[h]);
      else load8<T, false>(at, left, v[h]);
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = KMAJOR ? threadIdx.x / 4 + 64 * h : threadIdx.x / 16 + 16 * h;
      const int g = KMAJOR ? threadIdx.x % 4 : threadIdx.x % 16;
      unsigned char* at = lds + offset(r, g);
      if constexpr (PLANES == 3) {
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
      } else {
        *reinterpret_cast<uint4*>(at) = make_uint4(pack2_bf16(v[h][0], v[h][1]), pack2_bf16(v[h][2], v[h][3]), pack2_bf16(v[h][4], v[h][5]), pack2_bf16(v[h][6], v[h][7]));
      }
    }
  }
  // Granules of eight elements are exchanged within a row so that the lanes of a read fall into different banks: rows of 64 bytes (k-major), read
  // sixteen rows at a time, and of 256, read with eight sum indices at a time.
  __device__ static __forceinline__ int swap_of(int r) { return KMAJOR ? (r >> 2) & 3 : ((r & 3) | ((r >> 3) & 1) << 2) << 1; }
  __device__ static __forceinline__ int offset(int r, int granule) { return r * (KMAJOR ? RK * 2 : RT * 2) + (granule ^ swap_of(r)) * 16; }

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

// four neighbouring outputs of one row
template <typename C>
__device__ __forceinline__ void store_four(C* p, int left, const float (&v)[4], bool vec) {
  if (vec && left >= 4) {
    if constexpr (sizeof(C) == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = from_float<C>(v[i]);
  }
}

template <typename T, int KIND>
__global__ __launch_bounds__(256, 2) void linear_any_kernel(LinearArgs q) {
  typedef Staged<T, KIND != WGRAD> SA;
  typedef Staged<T, KIND == FORWARD> SB;
  typedef typename std::conditional<KIND == WGRAD, float, T>::type C;
  constexpr int P = SA::PLANES;
  __shared__ __align__(16) unsigned char lds[2 * P * RT * RK * 2];
  unsigned char *la = lds, *lb = lds + P * RT * RK * 2;

  const int n_tiles = (q.n + RT - 1) / RT, n0 = (int)(blockIdx.x % n_tiles) * RT;
  int group, m0, m_end, k_begin = 0, k_end = q.k;
  if (KIND == WGRAD) {
    const int m_tiles = (q.m + RT - 1) / RT, t = blockIdx.x / n_tiles;
    group = t / m_tiles;
    m0 = t % m_tiles * RT;
    m_end = q.m;
    group_rows(q.offs, q.groups, q.rows, group, k_begin, k_end);
  } else {
    if (!find_tile(q.offs, q.groups, q.rows, RT, blockIdx.x / n_tiles, group, m0, m_end)) return;
    if (group == q.groups) k_end = 0;                             // rows of no expert: zeros
  }
  const T* a = (const T*)q.a;
  const T* b = (const T*)q.b + (KIND == WGRAD ? 0 : (long long)(group < q.groups ? group : 0) * q.b_group);
  C* c = (C*)q.c + (KIND == WGRAD ? (long long)group * q.c_group : 0);

  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  floatx4 acc[4][4], low[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = low[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  SA sa;
  SB sb;
  if (k_begin < k_end) {
    sa.load(a, q.a_stride, m0, m_end, k_begin, k_end, q.vec & 1);
    sb.load(b, q.b_stride, n0, q.n, k_begin, k_end, q.vec & 2);
  }
  for (int k0 = k_begin; k0 < k_end; k0 += RK) {
    __syncthreads();
    sa.store(la);
    sb.store(lb);
    __syncthreads();
    if (k0 + RK < k_end) {
      sa.load(a, q.a_stride, m0, m_end, k0 + RK, k_end, q.vec & 1);
      sb.load(b, q.b_stride, n0, q.n, k0 + RK, k_end, q.vec & 2);
    }
    u32x4 fa[4][P];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) fa[i][p] = SA::read(la + p * SA::PLANE, wm + i * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4 fb[P];
#pragma unroll
      for (int p = 0; p < P; ++p) fb[p] = SB::read(lb + p * SB::PLANE, wn + j * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {                               // (b first: a lane then holds four neighbouring columns of one row)
        mma(acc[i][j], fb[0], fa[i][0]);
        if constexpr (P == 3) {
          mma(low[i][j], fb[0], fa[i][1]);
          mma(low[i][j], fb[1], fa[i][0]);
          mma(low[i][j], fb[1], fa[i][1]);
          mma(low[i][j], fb[0], fa[i][2]);
          mma(low[i][j], fb[2], fa[i][0]);
        }
      }
    }
  }

  bool again = false;                                             // fp32: a value out of the parts' range, an infinity or NaN
  if constexpr (P == 3) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i][j] = (acc[i][j] + low[i][j]) * SPLIT_UNSCALE;
#pragma unroll
        for (int e = 0; e < 4; ++e) again |= !finite_bits(__float_as_uint(acc[i][j][e]) & 0x7fffffffu);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + wm + i * 16 + (l & 15);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + j * 16 + (l >> 4) * 4;
      if (m >= m_end || n >= q.n) continue;
      float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
      if (again) {                                                // this lane's outputs as chains of fp32 multiply-adds
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (n + e >= q.n) continue;
          float sum = 0.f;
          for (int k = k_begin; k < k_end; ++k) {
            const float x = to_float(KIND == WGRAD ? a[(long long)k * q.a_stride + m] : a[(long long)m * q.a_stride + k]);
            const float y = to_float(KIND == FORWARD ? b[(long long)(n + e) * q.b_stride + k] : b[(long long)k * q.b_stride + n + e]);
            sum = fmaf(x, y, sum);
          }
          v[e] = sum;
        }
      }
      store_four<C>(c + (long long)m * q.c_stride + n, q.n - n, v, q.vec & 4);
    }
  }
}


// ---- rows of multiples of 16 bytes: bf16, and 8 bits ----
//
// Tiles of BM x BN, 64 of the sum's index a step, in LDS as bf16: k-major operands in rows of 128 bytes, the others as 64 rows (sum indices) of BM or BN
// values that are read with transposing reads.  bf16 operands are copied straight from memory while the step before the last is multiplied; 8-bit ones go through
// registers, where a code times its block's power of two becomes the bf16 number that it is: every product is exact and every sum fp32.
// (The 8-bit MFMAs would take half the matrix-pipe time, but they add eight neighbouring products with what lies 2^-13 below the largest of them
// cut off (2^16 + 2^2 is 2^16): 1.5e-5 of the result's norm on normal values, 5e-5 on codes of all sizes.)
constexpr int STEP = 64;

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

// A bf16 operand: copies.
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

// An 8-bit operand, k-major: chunks of sixteen codes of a row, thread t's being chunk t % 4 of rows t / 4, t / 4 + THREADS / 4, ...  A chunk is written to LDS two
// steps after it was asked for.
template <int R, int NW>
struct Converted : Tile<true, R, NW> {
  typedef Tile<true, R, NW> S;
  typedef uint8_t T;
  static constexpr bool COPIES = false;
  static constexpr int CHUNKS = R * 4 / (64 * NW);
  static constexpr int PIECES = CHUNKS;
  static_assert(R * 4 % (64 * NW) == 0, "whole chunks");
  uint4 q[CHUNKS];
  int byte[CHUNKS];
  __amdgpu_buffer_rsrc_t codes, scales;
  unsigned off[CHUNKS], scale_off[CHUNKS];
  int k;                                                          // of the step that is asked for next

  __device__ __forceinline__ void prepare(const T* base, const uint8_t* scale, long long stride, int row0, int rows, int k0, int k_end, int) {
    const long long blocks = stride / BLOCK8;
    codes = buffer_of(base + row0 * stride, (unsigned long long)(rows * stride));
    scales = buffer_of(scale + row0 * blocks, (unsigned long long)(rows * blocks));
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const int r = threadIdx.x / 4 + p * (16 * NW);
      off[p] = r < rows ? (unsigned)(r * stride) + threadIdx.x % 4 * 16 : NO_ROW;
      scale_off[p] = r < rows ? (unsigned)(r * blocks) : NO_ROW;
    }
    k = 0;
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) ask(p);
    k = STEP;
  }
  __device__ __forceinline__ void ask(int p) {
    // (behind the last step: the start of the rows again, which is not used)
    q[p] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)off[p], k, 0));
    byte[p] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)scale_off[p], k / BLOCK8, 0);
  }
  __device__ __forceinline__ void next_step() {}
  __device__ __forceinline__ void piece(int p, int, int left, unsigned char* lds, unsigned) {
    const int r = threadIdx.x / 4 + p * (16 * NW), c = threadIdx.x % 4 * 2;
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
    if (p == CHUNKS - 1) k = left > 2 * STEP ? k + STEP : 0;
  }
};

// One tile of expert `group` (q.groups: of none): rows m0 .. m_end - 1, columns n0 .., sum indices k_begin .. k_end - 1.
template <bool EIGHT, int KIND, int BM, int BN, int WM, int WN, typename C>
__device__ __forceinline__ void tile_product(const LinearArgs& q, unsigned char* lds, int group, int m0, int m_end, int n0, int k_begin, int k_end) {
  constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  typedef typename std::conditional<EIGHT, Converted<BM, NW>, Copied<KIND != WGRAD, BM, NW>>::type CA;
  typedef typename std::conditional<EIGHT, Converted<BN, NW>, Copied<KIND == FORWARD, BN, NW>>::type CB;
  typedef typename CA::T T;
  constexpr int STAGE = CA::BYTES + CB::BYTES;                    // two of them
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const int steps = (k_end - k_begin + STEP - 1) / STEP;
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
    const unsigned lds0 = lds_address(lds);
    constexpr int PIECES = CA::PIECES + CB::PIECES;
    auto copy_piece = [&](int p, int stage) {
      if (p < CA::PIECES) ca.piece(p, wave, left, lds + stage * STAGE, lds0 + stage * STAGE);
      else cb.piece(p - CA::PIECES, wave, left, lds + stage * STAGE + CA::BYTES, lds0 + stage * STAGE + CA::BYTES);
    };

    // Half a step is multiplied while the operands of the next half are read from LDS, so that the matrix pipe sees no wait: the second half's during the
    // first, and during the second those of the next step, whose copies have then had a whole step to arrive.  The barrier between the halves
    // says that they have, and that no wave reads this step's stage any more, which the copies of the step after the next overwrite.
    struct Operands { u32x4 a[TM], b[TN]; };
    Operands f0, f1;
    auto read_piece = [&](Operands& f, int p, int stage, int h) {
      const unsigned char* at = lds + stage * STAGE;
      if (p < TN) f.b[p] = CB::read(at + CA::BYTES, wn + p * 16, h);
      else f.a[p - TN] = CA::read(at, wm + (p - TN) * 16, h);
    };
    constexpr int SLOTS = TM > 2 ? TM - 1 : TM;                   // rows of products that reads and copies are issued between
    // products of `f`; meanwhile the operands `next` of half h of `stage`, and (COPY) the copies of another step into the other stage
    auto half_step = [&](const Operands& f, Operands& next, int stage, int h, auto copy) {
      static_for<0, TM>([&](auto iv) {
        constexpr int i = iv.value;
        static_for<i * (TM + TN) / SLOTS, (i + 1) * (TM + TN) / SLOTS>([&](auto p) { if constexpr (p.value < TM + TN) read_piece(next, p.value, stage, h); });
        if constexpr (copy.value)
          static_for<i * PIECES / SLOTS, (i + 1) * PIECES / SLOTS>([&](auto p) { if constexpr (p.value < PIECES) copy_piece(p.value, stage ^ 1); });
#pragma unroll
        for (int j = 0; j < TN; ++j) mma(acc[i][j], f.b[j], f.a[i]);
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    // (Copies behind the last step ask for nothing and fill the stage with zeros; its operands are read and not multiplied.)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      ca.next_step();
      cb.next_step();
#pragma unroll
      for (int p = 0; p < PIECES; ++p) copy_piece(p, s);
      left -= STEP;
    }
    if constexpr (CA::COPIES) wait_vm<0>();
    __syncthreads();
    static_for<0, TM + TN>([&](auto p) { read_piece(f0, p.value, 0, 0); });
    for (int s = 0; s < steps; ++s) {
      const int stage = s & 1;
      half_step(f0, f1, stage, 1, std::false_type());
      if constexpr (CA::COPIES) wait_vm<0>();
      __syncthreads();
      ca.next_step();
      cb.next_step();
      half_step(f1, f0, stage ^ 1, 0, std::true_type());
      left -= STEP;
    }
    if constexpr (CA::COPIES) wait_vm<0>();
    __syncthreads();                                              // nothing is written to LDS any more, or read
  }

  // Sixteen rows of a wave's columns at a time go through LDS, so that its lanes store whole rows, 16 bytes each: 64 lanes with four columns each of
  // sixteen rows would write 32 or 64 bytes of a row at a time, at 2.5 TB/s.
  C* c = (C*)q.c + (KIND == WGRAD ? (long long)group * q.c_group : 0);
  constexpr int WIDE = TN * 16 * (int)sizeof(C), LANES = WIDE / 16, EACH = 16 / (int)sizeof(C);
  unsigned char* out = lds + wave * 16 * (WIDE + 16);
  static_assert(NW * 16 * (WIDE + 16) <= 2 * STAGE && 64 % LANES == 0, "the outputs' LDS");
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if (m0 + wm + i * 16 >= m_end) break;
    if (q.vec & 4) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        store_four<C>((C*)(out + (l & 15) * (WIDE + 16)) + j * 16 + (l >> 4) * 4, 4, v, true);
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = l / LANES; r < 16; r += 64 / LANES) {
        const int m = m0 + wm + i * 16 + r, n = n0 + wn + l % LANES * EACH;
        const uint4 v = *reinterpret_cast<const uint4*>(out + r * (WIDE + 16) + l % LANES * 16);
        if (m >= m_end || n >= q.n) continue;
        C* at = c + (long long)m * q.c_stride + n;
        if (n + EACH <= q.n) {
          *reinterpret_cast<uint4*>(at) = v;
        } else {
          const C* e = reinterpret_cast<const C*>(out + r * (WIDE + 16) + l % LANES * 16);
          for (int k = 0; k < q.n - n; ++k) at[k] = e[k];
        }
      }
      __builtin_amdgcn_wave_barrier();
    } else {
      const int m = m0 + wm + i * 16 + (l & 15);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int n = n0 + wn + j * 16 + (l >> 4) * 4;
        if (m >= m_end || n >= q.n) continue;
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        store_four<C>(c + (long long)m * q.c_stride + n, q.n - n, v, false);
      }
    }
  }
}

// Rows of tiles in bands of 8, columns by 4 within a band: 32 tiles in a row, which the CUs of one XCD work on together, then read 8 + 4
// panels through its L2 in place of 64.
__device__ __forceinline__ void banded(unsigned id, unsigned row_tiles, unsigned col_tiles, unsigned& r, unsigned& c) {
  const unsigned band = id / (8 * col_tiles), first = band * 8, high = min(8u, row_tiles - first), in_band = id - first * col_tiles;
  const unsigned four = in_band / (high * 4), in_four = in_band - four * (high * 4);
  r = first + in_four % high;
  c = four * 4 + in_four / high;
}

// Forward and dgrad.  Block b runs on XCD b % 8: each XCD takes one stretch of the whole tiles, then its share of the experts' shorter last ones, in
// half the height where that is enough.
template <bool EIGHT, int KIND, int BM, int BN, int WM, int WN, typename C>
__global__ __launch_bounds__(64 * WM * WN) void linear_kernel(LinearArgs q) {
  extern __shared__ __align__(1024) unsigned char lds[];
  unsigned whole, ends;
  count_tiles(q.offs, q.groups, q.rows, BM, whole, ends);
  const unsigned cols = (unsigned)(q.n + BN - 1) / BN, xcd = blockIdx.x & 7, i = blockIdx.x >> 3, share = (whole * cols + 7) / 8;
  int group, m0, m_end;
  if (i < share) {
    const unsigned id = xcd * share + i;
    if (id >= whole * cols) return;
    unsigned r, c;
    banded(id, whole, cols, r, c);
    find_tile_of<false>(q.offs, q.groups, q.rows, BM, r, group, m0, m_end);
    tile_product<EIGHT, KIND, BM, BN, WM, WN, C>(q, lds, group, m0, m_end, (int)c * BN, 0, group < q.groups ? q.k : 0);
  } else {
    const unsigned id = (i - share) * 8 + xcd;
    if (id >= ends * cols) return;
    find_tile_of<true>(q.offs, q.groups, q.rows, BM, id / cols, group, m0, m_end);
    const int n0 = (int)(id % cols) * BN, k = group < q.groups ? q.k : 0;
    if (m_end - m0 > BM / 2) tile_product<EIGHT, KIND, BM, BN, WM, WN, C>(q, lds, group, m0, m_end, n0, 0, k);
    else tile_product<EIGHT, KIND, BM / 2, BN, WM, WN, C>(q, lds, group, m0, m_end, n0, 0, k);
  }
}

template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void linear_wgrad_kernel(LinearArgs q) {
  extern __shared__ __align__(1024) unsigned char lds[];
  const int n_tiles = (q.n + BN - 1) / BN, m_tiles = (q.m + BM - 1) / BM, t = blockIdx.x / n_tiles;
  int begin, end;
  group_rows(q.offs, q.groups, q.rows, t / m_tiles, begin, end);
  tile_product<false, WGRAD, BM, BN, WM, WN, float>(q, lds, t / m_tiles, t % m_tiles * BM, q.m, (int)(blockIdx.x % n_tiles) * BN, begin, end);
}

// ---- launches ----

constexpr long long MOST_BLOCKS = 0x7fffffff;

template <typename T>
gan_status launch_any(int kind, const LinearArgs& q, hipStream_t st) {
  const long long n_tiles = (q.n + RT - 1) / RT;
  const long long blocks = n_tiles * (kind == WGRAD ? (long long)q.groups * ((q.m + RT - 1) / RT) : most_tiles(q.rows, q.groups, RT));
  if (blocks > MOST_BLOCKS) return operator_fail(GAN_E_SHAPE, "more than 2^31 - 1 tiles");
  const dim3 grid((unsigned)blocks), block(256);
  if (kind == FORWARD) hipLaunchKernelGGL((linear_any_kernel<T, FORWARD>), grid, block, 0, st, q);
  else if (kind == DGRAD) hipLaunchKernelGGL((linear_any_kernel<T, DGRAD>), grid, block, 0, st, q);
  else hipLaunchKernelGGL((linear_any_kernel<T, WGRAD>), grid, block, 0, st, q);
  return operator_launched();
}

template <typename F>
gan_status launch(F* kernel, long long blocks, int threads, int lds, const LinearArgs& q, hipStream_t st) {
  if (blocks > MOST_BLOCKS) return operator_fail(GAN_E_SHAPE, "more than 2^31 - 1 tiles");
  if (lds > 65536 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) {
    (void)hipGetLastError();
    return operator_fail(GAN_E_HIP, "the kernel's LDS could not be set");
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), lds, st, q);
  return operator_launched();
}

template <bool EIGHT, int KIND, int BM, int BN, int WM, int WN, typename C>
gan_status launch_tiles(const LinearArgs& q, hipStream_t st) {
  const long long cols = (q.n + BN - 1) / BN;
  constexpr int LDS = 2 * (BM + BN) * 128;
  if constexpr (KIND == WGRAD)
    return launch(linear_wgrad_kernel<BM, BN, WM, WN>, q.groups * cols * ((q.m + BM - 1) / BM), 64 * WM * WN, LDS, q, st);
  else    // (whole tiles and ends are each shared among the eight XCDs)
    return launch(linear_kernel<EIGHT, KIND, BM, BN, WM, WN, C>, 8 * ((most_tiles(q.rows, q.groups, BM) * cols + 7) / 8 + 1), 64 * WM * WN, LDS, q, st);
}

template <bool EIGHT, int KIND, typename C>
gan_status launch_aligned(const LinearArgs& q, hipStream_t st) {
  return launch_tiles<EIGHT, KIND, 256, 256, 2, 4, C>(q, st);
}

gan_status check(int32_t precision, const void* x, const void* w, const int32_t* offs, int32_t groups, int64_t rows, int32_t n_in, int32_t n_out, const void* out) {
  if (precision != GAN_FP32 && precision != GAN_BF16_FP32MASTER) return operator_fail(GAN_E_ARG, "unknown precision");
  if (!x || !w || !offs || !out) return operator_fail(GAN_E_ARG, "an operand is NULL");
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
  if (const gan_status s = check(precision, x, w, offs, groups, rows, n_in, n_out, y)) return s;
  if (x_stride < n_in || y_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or y_stride below n_out");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool va = rows_aligned16(x, x_stride, e) && n_in % 8 == 0, vb = rows_aligned16(w, n_in, e) && n_in % 8 == 0;
  const LinearArgs q = {x, w, nullptr, nullptr, y, offs, x_stride, n_in, y_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_out, n_in,
                        (va ? 1 : 0) | (vb ? 2 : 0) | (rows_aligned16(y, y_stride, e) ? 4 : 0)};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (precision == GAN_FP32) return launch_any<float>(FORWARD, q, st);
  return va && vb && short_rows(x_stride, e) && short_rows(n_in, e) ? launch_aligned<false, FORWARD, bf16_t>(q, st) : launch_any<bf16_t>(FORWARD, q, st);
}

extern "C" gan_status gan_group_linear_dgrad(int32_t precision, const void* dy, int64_t dy_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                             int32_t n_in, int32_t n_out, void* dx, int64_t dx_stride, void* hip_stream) {
  if (const gan_status s = check(precision, dy, w, offs, groups, rows, n_in, n_out, dx)) return s;
  if (dy_stride < n_out || dx_stride < n_in) return operator_fail(GAN_E_ARG, "dy_stride is below n_out, or dx_stride below n_in");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool va = rows_aligned16(dy, dy_stride, e) && n_out % 8 == 0, vb = rows_aligned16(w, n_in, e) && n_in % 8 == 0;
  const LinearArgs q = {dy, w, nullptr, nullptr, dx, offs, dy_stride, n_in, dx_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_in, n_out,
                        (va ? 1 : 0) | (vb ? 2 : 0) | (rows_aligned16(dx, dx_stride, e) ? 4 : 0)};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (precision == GAN_FP32) return launch_any<float>(DGRAD, q, st);
  return va && vb && short_rows(dy_stride, e) && short_rows(n_in, e) ? launch_aligned<false, DGRAD, bf16_t>(q, st) : launch_any<bf16_t>(DGRAD, q, st);
}

extern "C" int64_t gan_group_linear_wgrad_bytes(int32_t groups, int64_t rows, int32_t n_in, int32_t n_out) {
  return 0;
}

extern "C" gan_status gan_group_linear_wgrad(int32_t precision, const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, const int32_t* offs,
                                             int32_t groups, int64_t rows, int32_t n_in, int32_t n_out, float* dw, void* work, int64_t work_bytes, void* hip_stream) {
  if (const gan_status s = check(precision, x, dy, offs, groups, rows, n_in, n_out, dw)) return s;
  if (x_stride < n_in || dy_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or dy_stride below n_out");
  if (work_bytes < gan_group_linear_wgrad_bytes(groups, rows, n_in, n_out) || !aligned16(work))
    return operator_fail(GAN_E_ARG, "work is smaller than gan_group_linear_wgrad_bytes, or not 16-byte aligned");
  if (groups == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool va = rows_aligned16(dy, dy_stride, e) && n_out % 8 == 0, vb = rows_aligned16(x, x_stride, e) && n_in % 8 == 0;
  const LinearArgs q = {dy, x, nullptr, nullptr, dw, offs, dy_stride, x_stride, n_in, 0, (long long)n_in * n_out, groups, (int)rows, n_out, n_in, 0,
                        (va ? 1 : 0) | (vb ? 2 : 0) | (rows_aligned16(dw, n_in, 4) ? 4 : 0)};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (precision == GAN_FP32) return launch_any<float>(WGRAD, q, st);
  return va && vb && short_rows(x_stride, e) && short_rows(dy_stride, e) ? launch_aligned<false, WGRAD, float>(q, st) : launch_any<bf16_t>(WGRAD, q, st);
}

extern "C" gan_status gan_group_linear8(const uint8_t* x8, const uint8_t* x_scale, const uint8_t* w8, const uint8_t* w_scale, const int32_t* offs, int32_t groups,
                                        int64_t rows, int32_t n_in, int32_t n_out, int32_t y_precision, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(y_precision, x8, w8, offs, groups, rows, n_in, n_out, y)) return s;
  if (!x_scale || !w_scale) return operator_fail(GAN_E_ARG, "x_scale or w_scale is NULL");
  if (!aligned16(x8) || !aligned16(w8)) return operator_fail(GAN_E_ARG, "x8 or w8 is not 16-byte aligned");
  if (y_stride < n_out) return operator_fail(GAN_E_ARG, "y_stride is below n_out");
  const long long k = padded8(n_in);
  if (!short_rows(k, 1)) return operator_fail(GAN_E_SHAPE, "more than 2^22 inputs in 8 bits");
  if (rows == 0) return GAN_OK;
  const int e = y_precision == GAN_FP32 ? 4 : 2;
  const LinearArgs q = {x8, w8, x_scale, w_scale, y, offs, k, k, y_stride, k * n_out, 0, groups, (int)rows, 0, n_out, (int)k,
                        rows_aligned16(y, y_stride, e) ? 7 : 3};
  const hipStream_t st = (hipStream_t)hip_stream;
  return y_precision == GAN_FP32 ? launch_aligned<true, FORWARD, float>(q, st) : launch_aligned<true, FORWARD, bf16_t>(q, st);
}
