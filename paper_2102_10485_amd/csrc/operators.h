// What the operators for label experts share: refusals, the 8-bit format, vectors of eight elements.
#pragma once

#include "../../include/gan.h"
#include "common.h"

namespace gan {

gan_status operator_fail(gan_status s, const char* why);          // records the calling thread's text and returns s
void operator_launches();                                         // before a launch: what an earlier HIP call of the caller's left behind is not its failure
gan_status operator_launched();                                   // GAN_OK, or GAN_E_HIP with the runtime's text

constexpr long long PAST_CACHES = 64 << 20;                      // bytes of a result that its reader would not find in the caches
constexpr long long MOST_ROWS = 1 << 30;
constexpr int MOST_COLS = 1 << 28;
gan_status check_sizes(int32_t precision, long long rows, int cols);
gan_status check_matrix(const void* p, long long stride, int cols, const char* why);

constexpr int BLOCK8 = 128;                                       // neighbours that share a scale
__host__ __device__ inline long long padded8(long long cols) { return (cols + BLOCK8 - 1) / BLOCK8 * BLOCK8; }

// Eight neighbouring elements as fp32, from 16-byte aligned memory (VEC, where none or all eight are left) or any; one by one
// where fewer than eight are left.  What is missing is zero.
template <int ALIGN> struct Words;
template <> struct Words<16> { typedef unsigned T __attribute__((ext_vector_type(4))); };
template <> struct Words<4> { typedef unsigned T __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Words<2> { typedef unsigned T __attribute__((ext_vector_type(4), aligned(2))); };

template <typename T, int ALIGN>
__device__ __forceinline__ void load_whole8(const T* p, float (&v)[8]) {
  typedef typename Words<ALIGN>::T words;
  const words a = reinterpret_cast<const words*>(p)[0];
  if constexpr (sizeof(T) == 4) {
    const words b = *reinterpret_cast<const words*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __uint_as_float(a[i]);
      v[4 + i] = __uint_as_float(b[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int left, float (&v)[8]) {
  if constexpr (VEC) {
    if (left <= 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
      load_whole8<T, 16>(p, v);
    }
  } else {
    if (left >= 8) {
      load_whole8<T, sizeof(T)>(p, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? to_float(p[i]) : 0.f;
    }
  }
}

// Eight neighbours as they lie in memory, to be had in flight in few registers: read as load8 does, values later.
template <typename T>
struct Raw8 {
  unsigned w[2 * sizeof(T)];
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p, int left) {
    typedef typename Words<VEC ? 16 : sizeof(T)>::T words;
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) w[i] = 0;
    if (VEC ? left > 0 : left >= 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const words v = reinterpret_cast<const words*>(p)[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
      }
    } else if (!VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = i < left ? __float_as_uint(p[i]) : 0u;
        else w[i / 2] |= (i < left ? (unsigned)p[i].v : 0u) << 16 * (i % 2);
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = sizeof(T) == 4 ? __uint_as_float(w[i % (2 * sizeof(T))]) : __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  template <bool VEC, bool PAST = false>
  __device__ __forceinline__ void store(T* p, int left) const {
    typedef typename Words<VEC ? 16 : sizeof(T)>::T words;
    if (VEC ? left > 0 : left >= 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const words v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<words*>(p) + i);
        else reinterpret_cast<words*>(p)[i] = v;
      }
    } else if (!VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) { if (i < left) p[i] = __uint_as_float(w[i]); }
        else { if (i < left) p[i].v = (unsigned short)(w[i / 2] >> 16 * (i % 2)); }
      }
    }
  }
};

// PAST: past the caches
template <typename T, int ALIGN, bool PAST>
__device__ __forceinline__ void store_whole8(T* p, const float (&v)[8]) {
  typedef typename Words<ALIGN>::T words;
  words* to = reinterpret_cast<words*>(p);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    words w;
    if constexpr (sizeof(T) == 4) w = words{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
    else w = words{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
    if constexpr (PAST) __builtin_nontemporal_store(w, to + i);
    else to[i] = w;
  }
}
template <typename T, bool VEC, bool PAST = false>
__device__ __forceinline__ void store8(T* p, int left, const float (&v)[8]) {
  if constexpr (VEC) {
    if (left > 0) store_whole8<T, 16, PAST>(p, v);
  } else if (left >= 8) {
    store_whole8<T, sizeof(T), PAST>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = from_float<T>(v[i]);
  }
}

template <bool PAST>
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 q) {                // eight of them, aligned
  const uint64_t w = q.x | (uint64_t)q.y << 32;
  if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<uint64_t*>(p));
  else *reinterpret_cast<uint64_t*>(p) = w;
}

// ---- the 8-bit format: e4m3 times one power of two for 128 neighbours, which 16 lanes hold, eight each ----

__device__ __forceinline__ bool finite_bits(unsigned magnitude) { return magnitude < 0x7f800000u; }

// The block's scale byte E + 127: the least E in [-126, 127] with every finite |value| <= 448 * 2^E = 1.75 * 2^(E+8).  The bits of the largest
// magnitude carry into the exponent where its mantissa is above 1.75.
__device__ __forceinline__ int scale_byte(const float (&v)[8]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned a = __float_as_uint(v[i]) & 0x7fffffffu;
    top = max(top, finite_bits(a) ? a : 0u);
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) top = max(top, (unsigned)__shfl_xor((int)top, d));
  return max((int)((top + 0x1fffffu) >> 23) - 8, 1);
}
__device__ __forceinline__ float power_of_two(int biased) { return __uint_as_float((unsigned)biased << 23); }    // biased in [1, 254]; 0 gives 0

// Rounded to nearest even.  Scaled values are within +-448, where the conversion needs no saturation.
__device__ __forceinline__ unsigned to_e4m3_x4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ uint2 to_e4m3_x8(const float (&v)[8], int byte) {
  const float f = power_of_two(254 - byte);
  float s[8];
  unsigned bad = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s[i] = v[i] * f;
    bad |= (finite_bits(__float_as_uint(v[i]) & 0x7fffffffu) ? 0u : 1u) << i;
  }
  uint2 q = make_uint2(to_e4m3_x4(s[0], s[1], s[2], s[3]), to_e4m3_x4(s[4], s[5], s[6], s[7]));
  if (bad) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (bad >> i & 1) {
        unsigned& w = i < 4 ? q.x : q.y;
        w = (w & ~(0xffu << 8 * (i & 3))) | 0x7fu << 8 * (i & 3);
      }
  }
  return q;
}
__device__ __forceinline__ void from_e4m3_x8(uint2 q, int byte, float (&v)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const float f = power_of_two(byte);
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, true);
  v[0] = a.x * f; v[1] = a.y * f; v[2] = b.x * f; v[3] = b.y * f;
  v[4] = c.x * f; v[5] = c.y * f; v[6] = d.x * f; v[7] = d.y * f;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// whether rows of this matrix start at multiples of 16 bytes (no matrix: yes)
inline bool rows_aligned16(const void* p, long long stride, int esize) { return aligned16(p) && stride * esize % 16 == 0; }

}  // namespace gan
