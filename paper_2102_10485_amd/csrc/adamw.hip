// AdamW over many tensors in one launch, with moments in 32 bits or in 8.
//
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: 30 bytes a value with fp32 gradients, fp32 moments and the bf16 copy, 16 with bf16 gradients, moments of 8 bits and the copy.  A
// hundred million values on an MI355X: 551 us and 298 us, 5.4 TB/s both (a plain copy: 4.9 of reads and writes); 210 million in four tensors, 8 bits: 613 us.
// A block takes CHUNK values of one tensor; which ones it reads off a table that the handle laid out once, so that small and
// large tensors share the launch.  In 8 bits the moments of 128 values, which sixteen lanes hold, share a power of two (operators.h): m as it is and the
// square root of v, whose range is half of v's.  Both are rounded by chance: with b2 = 0.999 a step moves sqrt(v) by 0.05 % of its distance
// from |g|, far below half a code (6 %), so that rounding to nearest would hold v for ever.
#include <math.h>

#include <new>
#include <vector>

#include "operators.h"

namespace gan {
namespace {

constexpr int E = 8, CHUNK = 2048;

struct Tensor {
  float* p;
  const void* g;
  bf16_t* copy;                // or NULL
  long long size, first;       // values; index of the first one in the moments
  float decay;
  int vec;                     // p, g and copy are 16-byte aligned
};
struct Chunk {
  int tensor, at;              // the at'th CHUNK of it
};

struct StepArgs {
  const Tensor* tensors;
  const Chunk* chunks;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  float lr, b1, one_minus_b1, b2, one_minus_b2, root_factor, eps, step_size;
  unsigned key;
};

// 32 well-mixed bits of an index: two rounds of a shift and a product modulo 2^32 (odd factors, the digits of sqrt(2) and sqrt(3))
__device__ __forceinline__ unsigned mixed(unsigned long long i, unsigned key) {
  unsigned u = ((unsigned)i + (unsigned)(i >> 32) * 0x9E3779B9u) ^ key;
  u = (u ^ u >> 16) * 0x6A09E667u;
  u = (u ^ u >> 15) * 0xBB67AE85u;
  return u ^ u >> 16;
}

// e4m3 magnitude of a = |x| * 2^-E <= 448: floor(a / ulp + u) with u in [0, 1) in steps of 2^-16; the lowest binade and what is
// below it share an ulp
__device__ __forceinline__ unsigned e4m3_by_chance(float a, unsigned u16) {
  const int binade = min(max((int)(__float_as_uint(a) >> 23), 121), 135);
  const float t = a * __uint_as_float((unsigned)(257 - binade) << 23);
  return (unsigned)((binade - 121) * 8 + (int)floorf(__fadd_rn(t, (float)u16 * 0x1p-16f)));
}

template <bool NEVER_ZERO>
__device__ __forceinline__ uint2 encode8(const float (&x)[E], int byte, const unsigned (&u)[E]) {
  const float f = power_of_two(254 - byte);
  unsigned q[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const unsigned bits = __float_as_uint(x[i]);
    const float a = fabsf(x[i]) * f;
    unsigned code = e4m3_by_chance(a, NEVER_ZERO ? u[i] >> 16 : u[i] & 0xffffu);
    if (NEVER_ZERO && code == 0 && a > 0.f) code = 1;
    code = finite_bits(bits & 0x7fffffffu) ? code | bits >> 31 << 7 : 0x7f;
    q[i / 4] |= code << 8 * (i % 4);
  }
  return make_uint2(q[0], q[1]);
}

// Every operation is rounded on its own (none contracted into a multiply-add): the result is what the formula gives in
// any program that computes in fp32, and with it the codes.
template <typename G, bool EIGHT, bool VEC>
__device__ __forceinline__ void update8(const StepArgs& a, const Tensor& t, long long i) {
#pragma clang fp contract(off)
  const int left = (int)min((long long)E, t.size - i);
  const long long at = t.first + i;
  float p[E], g[E], m[E], v[E];
  load8<float, VEC>(t.p + i, left, p);
  load8<G, VEC>((const G*)t.g + i, left, g);
  if constexpr (EIGHT) {
    from_e4m3_x8(*reinterpret_cast<const uint2*>((const uint8_t*)a.m + at), a.m_scale[at / BLOCK8], m);
    from_e4m3_x8(*reinterpret_cast<const uint2*>((const uint8_t*)a.v + at), a.v_scale[at / BLOCK8], v);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = v[k] * v[k];
  } else {
    load8<float, true>((const float*)a.m + at, E, m);
    load8<float, true>((const float*)a.v + at, E, v);
  }
  const float keep = 1.f - t.decay * a.lr;
  float root[E];
#pragma unroll
  for (int k = 0; k < E; ++k) {
    m[k] = m[k] * a.b1 + g[k] * a.one_minus_b1;
    v[k] = v[k] * a.b2 + g[k] * g[k] * a.one_minus_b2;
    root[k] = sqrtf(v[k]);
    p[k] = p[k] * keep - m[k] / (root[k] * a.root_factor + a.eps) * a.step_size;
  }
  store8<float, VEC>(t.p + i, left, p);
  if (t.copy) store8<bf16_t, VEC>(t.copy + i, left, p);
  if constexpr (EIGHT) {
    unsigned u[E];
#pragma unroll
    for (int k = 0; k < E; ++k) u[k] = mixed((unsigned long long)at + k, a.key);
    const int mb = scale_byte(m), vb = scale_byte(root);
    *reinterpret_cast<uint2*>((uint8_t*)a.m + at) = encode8<false>(m, mb, u);
    *reinterpret_cast<uint2*>((uint8_t*)a.v + at) = encode8<true>(root, vb, u);
    if ((threadIdx.x & 15) == 0) {
      a.m_scale[at / BLOCK8] = (uint8_t)mb;
      a.v_scale[at / BLOCK8] = (uint8_t)vb;
    }
  } else {
    store8<float, true>((float*)a.m + at, E, m);
    store8<float, true>((float*)a.v + at, E, v);
  }
}

template <typename G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(StepArgs a) {
  const Chunk c = a.chunks[blockIdx.x];
  const Tensor t = a.tensors[c.tensor];
  const long long i = (long long)c.at * CHUNK + threadIdx.x * E;
  if (i >= (t.size + BLOCK8 - 1) / BLOCK8 * BLOCK8) return;        // (all of a block of 128 or none: its lanes share the scale)
  // whole vectors where the tensor is aligned; its last block one by one (all lanes of a block go the same way)
  if (t.vec && (i | (BLOCK8 - 1)) < t.size) update8<G, EIGHT, true>(a, t, i);
  else update8<G, EIGHT, false>(a, t, i);
}

}  // namespace
}  // namespace gan

using namespace gan;

struct gan_adamw {
  Tensor* tensors = nullptr;
  Chunk* chunks = nullptr;
  long long n_chunks = 0;
  int bf16_grads = 0, eight = 0;
  void *m = nullptr, *v = nullptr;
  uint8_t *m_scale = nullptr, *v_scale = nullptr;
  ~gan_adamw() {
    (void)hipFree(tensors);
    (void)hipFree(chunks);
  }
};

extern "C" int64_t gan_adamw_blocks(int32_t tensors, const int64_t* sizes) {
  if (tensors < 1 || !sizes) return 0;
  int64_t n = 0;
  for (int t = 0; t < tensors; ++t) {
    if (sizes[t] < 0 || sizes[t] > ((int64_t)1 << 40)) return 0;
    n += (sizes[t] + BLOCK8 - 1) / BLOCK8;
  }
  return n;
}

extern "C" gan_status gan_adamw_create(int32_t tensors, const int64_t* sizes, float* const* params, const void* const* grads, int32_t grad_precision,
                                       void* const* copies, const float* decay, int32_t state_bits, void* m, void* v, uint8_t* m_scale, uint8_t* v_scale,
                                       gan_adamw** out) {
  if (!out) return operator_fail(GAN_E_ARG, "out is NULL");
  *out = nullptr;
  if (tensors < 1 || !sizes || !params || !grads) return operator_fail(GAN_E_ARG, "no tensors, or sizes, params or grads is NULL");
  const bool any = gan_adamw_blocks(tensors, sizes) > 0;           // (tensors without values have no moments)
  if (any && (!m || !v)) return operator_fail(GAN_E_ARG, "m or v is NULL");
  if (grad_precision != GAN_FP32 && grad_precision != GAN_BF16_FP32MASTER) return operator_fail(GAN_E_ARG, "unknown precision");
  if (state_bits != 32 && state_bits != 8) return operator_fail(GAN_E_ARG, "state_bits is neither 32 nor 8");
  if (state_bits == 8 ? any && (!m_scale || !v_scale) : m_scale || v_scale)
    return operator_fail(GAN_E_ARG, "m_scale and v_scale go with state_bits 8");
  if (!aligned16(m) || !aligned16(v)) return operator_fail(GAN_E_ARG, "m or v is not 16-byte aligned");
  try {
    std::vector<Tensor> table;
    std::vector<Chunk> chunks;
    long long first = 0;
    for (int t = 0; t < tensors; ++t) {
      if (sizes[t] < 0 || sizes[t] > ((int64_t)1 << 40)) return operator_fail(GAN_E_ARG, "a tensor of negative size, or of more than 2^40 values");
      if (sizes[t] > 0 && (!params[t] || !grads[t])) return operator_fail(GAN_E_ARG, "an entry of params or grads is NULL");
      if (decay && !(decay[t] >= 0.f && decay[t] <= 3.4e38f)) return operator_fail(GAN_E_ARG, "a decay is negative or not finite");
      void* copy = copies ? copies[t] : nullptr;
      table.push_back({params[t], grads[t], (bf16_t*)copy, sizes[t], first, decay ? decay[t] : 0.f,
                       aligned16(params[t]) && aligned16(grads[t]) && aligned16(copy)});
      for (long long c = 0; c * CHUNK < sizes[t]; ++c) chunks.push_back({t, (int)c});
      first += (sizes[t] + BLOCK8 - 1) / BLOCK8 * BLOCK8;
    }
    if (chunks.size() > 0x7fffffffull) return operator_fail(GAN_E_SHAPE, "more than 2^42 values");
    gan_adamw* h = new gan_adamw;
    h->n_chunks = (long long)chunks.size();
    h->bf16_grads = grad_precision == GAN_BF16_FP32MASTER;
    h->eight = state_bits == 8;
    h->m = m; h->v = v; h->m_scale = m_scale; h->v_scale = v_scale;
    const size_t tb = table.size() * sizeof(Tensor), cb = chunks.size() * sizeof(Chunk);
    if (hipMalloc((void**)&h->tensors, tb) != hipSuccess || (cb && hipMalloc((void**)&h->chunks, cb) != hipSuccess)) {
      (void)hipGetLastError();
      delete h;
      return operator_fail(GAN_E_OOM, "no device memory for the table of tensors");
    }
    if (hipMemcpy(h->tensors, table.data(), tb, hipMemcpyHostToDevice) != hipSuccess ||
        (cb && hipMemcpy(h->chunks, chunks.data(), cb, hipMemcpyHostToDevice) != hipSuccess)) {
      (void)hipGetLastError();
      delete h;
      return operator_fail(GAN_E_HIP, "the table of tensors could not be copied to the device");
    }
    *out = h;
    return GAN_OK;
  } catch (...) {
    return operator_fail(GAN_E_OOM, "no host memory for the table of tensors");
  }
}

extern "C" gan_status gan_adamw_step(gan_adamw* h, double lr, double beta1, double beta2, double eps, int64_t step, uint32_t seed, void* hip_stream) {
  if (!h) return operator_fail(GAN_E_ARG, "no handle");
  if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && eps >= 0 && lr >= 0 && lr <= 1e30) || step < 1)
    return operator_fail(GAN_E_ARG, "a beta outside [0, 1), a negative eps or lr, or a step below 1");
  if (h->n_chunks == 0) return GAN_OK;
  StepArgs a;
  a.tensors = h->tensors;
  a.m = h->m; a.v = h->v; a.m_scale = h->m_scale; a.v_scale = h->v_scale;
  a.lr = (float)lr;
  a.b1 = (float)beta1; a.one_minus_b1 = (float)(1 - beta1);
  a.b2 = (float)beta2; a.one_minus_b2 = (float)(1 - beta2);
  a.root_factor = (float)(1 / sqrt(1 - pow(beta2, (double)step)));
  a.eps = (float)eps;
  a.step_size = (float)(lr / (1 - pow(beta1, (double)step)));
  a.key = seed + (unsigned)step * 0x9E3779B9u;
  const hipStream_t st = (hipStream_t)hip_stream;
  // a launch has fewer than 2^32 threads (the runtime takes more of them modulo 2^32, without an error): 2^23 chunks at a time
  constexpr long long MOST = 1 << 23;
  operator_launches();
  for (long long first = 0; first < h->n_chunks; first += MOST) {
    a.chunks = h->chunks + first;
    const dim3 grid((unsigned)(h->n_chunks - first < MOST ? h->n_chunks - first : MOST)), block(256);
    if (h->bf16_grads) {
      if (h->eight) hipLaunchKernelGGL((adamw_kernel<bf16_t, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((adamw_kernel<bf16_t, false>), grid, block, 0, st, a);
    } else {
      if (h->eight) hipLaunchKernelGGL((adamw_kernel<float, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((adamw_kernel<float, false>), grid, block, 0, st, a);
    }
  }
  return operator_launched();
}

extern "C" gan_status gan_adamw_destroy(gan_adamw* h) {
  if (!h) return GAN_OK;
  const bool ok = hipDeviceSynchronize() == hipSuccess;
  delete h;
  return ok ? GAN_OK : operator_fail(GAN_E_HIP, "the device's work did not end without an error");
}
