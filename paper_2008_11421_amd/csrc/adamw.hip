// AdamW over many tensors at once, moments in fp32 or in 8 bits:
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   w -= lr weight_decay w + lr c1 m / (k2 sqrt(v) + eps),  c1 = 1 / (1 - b1^step),  k2 = 1 / sqrt(1 - b2^step).
// 8 bits: blocks of 64 values share an fp32 scale s.  m = q s with q in -127 .. 127, v = q^2 s with q in 0 .. 255 (the
// square gives small second moments next to large ones four more bits than a linear code).  A value falls between two
// codes and goes to one of them at random, so that its expectation is the value itself: v changes by a thousandth of itself
// a step, and rounding to the nearest code would hold it where it is for good.  The random bits are a hash of the element's
// place and the call's seed.  v > 0 never becomes code 0: m over eps alone would be a huge step.
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

// The tensors of one launch: their descriptors travel as kernel arguments, 4 KB in all.
template <bool EIGHT>
struct AdamwTensor {
  float* w; void* m; void* v; const void* grad; void* out;
  size_t n;
  float decay;
  unsigned flags;
};
template <>
struct AdamwTensor<true> : AdamwTensor<false> {
  float* m_scale; float* v_scale;
  unsigned key;     // of the tensor's random bits, the seed aside
};
template <bool EIGHT>
struct AdamwSet {
  static constexpr int MOST = EIGHT ? 46 : 66;
  AdamwTensor<EIGHT> t[MOST];
  unsigned first[MOST + 1];     // tensor k has workgroups [first[k], first[k + 1])
  int n;
};
struct AdamwNow {
  float lr, beta1, beta2, eps, grad_scale;
  float c1, k2;                 // not with live
  unsigned seed;
  const karma_adamw_live* live;
};
static_assert(sizeof(AdamwSet<false>) + sizeof(AdamwNow) <= 4096 && sizeof(AdamwSet<true>) + sizeof(AdamwNow) <= 4096, "kernel arguments");

// the tensor of this workgroup
template <typename Set>
__device__ __forceinline__ int tensor_of(const Set& u) {
  int lo = 0, hi = u.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (blockIdx.x >= u.first[mid]) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// 1 - beta^step by repeated squaring: one rounding a multiplication, the same on the host and on the device
__host__ __device__ inline double one_minus_power(float beta, unsigned long long step) {
  double p = 1.0, b = beta;
  for (; step; step >>= 1, b *= b)
    if (step & 1) p *= b;
  return 1.0 - p;
}
__host__ __device__ inline void corrections(AdamwNow& a, unsigned long long step) {
  a.c1 = (float)(1.0 / one_minus_power(a.beta1, step));
  a.k2 = (float)(1.0 / sqrt(one_minus_power(a.beta2, step)));
}

__device__ __forceinline__ unsigned random_bits(unsigned long long i, unsigned key) {
  unsigned x = (unsigned)i + key;
  x = (x ^ (x >> 16)) * 0x45c3a2adu;
  x = (x ^ (x >> 15)) * 0x2d51f9b5u;
  return x ^ (x >> 16);
}

// The largest of 16 lanes' values, none of which is negative: as whole numbers they have the same order, and NaN is the largest.
__device__ __forceinline__ float max16(float v) {
  unsigned x = __float_as_uint(v);
#define KARMA_MAX_STEP(CTRL) x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false))
  KARMA_MAX_STEP(0xB1);     // quad_perm [1,0,3,2]
  KARMA_MAX_STEP(0x4E);     // quad_perm [2,3,0,1]
  KARMA_MAX_STEP(0x141);    // row_half_mirror
  KARMA_MAX_STEP(0x140);    // row_mirror
#undef KARMA_MAX_STEP
  return __uint_as_float(x);
}

// Four consecutive values of a buffer: at once where `whole` (all four exist and the buffer is aligned), else one by one.
typedef __attribute__((ext_vector_type(4))) float f32x4;
__device__ __forceinline__ f32x4 load4(const float* p, size_t i, size_t n, bool whole) {
  if (whole) return *(const f32x4*)(p + i);
  f32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = i + e < n ? p[i + e] : 0.f;
  return r;
}
__device__ __forceinline__ f32x4 load4(const bf16_t* p, size_t i, size_t n, bool whole) {
  f32x4 r;
  if (whole) {
    const u32x2 v = *(const u32x2*)(p + i);
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = i + e < n ? bf2f(p[i + e]) : 0.f;
  return r;
}
__device__ __forceinline__ unsigned load4(const uint8_t* p, size_t i, size_t n, bool whole) {
  if (whole) return *(const unsigned*)(p + i);
  unsigned r = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) r |= i + e < n ? (unsigned)p[i + e] << (8 * e) : 0u;
  return r;
}
__device__ __forceinline__ void store4(float* p, size_t i, size_t n, bool whole, const f32x4& v) {
  if (whole) { *(f32x4*)(p + i) = v; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (i + e < n) p[i + e] = v[e];
}
__device__ __forceinline__ void store4(bf16_t* p, size_t i, size_t n, bool whole, const f32x4& v) {
  if (whole) { *(u32x2*)(p + i) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])}; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (i + e < n) p[i + e] = f2bf(v[e]);
}
__device__ __forceinline__ void store4(uint8_t* p, size_t i, size_t n, bool whole, unsigned v) {
  if (whole) { *(unsigned*)(p + i) = v; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (i + e < n) p[i + e] = (uint8_t)(v >> (8 * e));
}

// 1 / s in 64 bits, 0 for 0: the hardware's approximation of 2^-26 and two Newton steps (a division takes three times as long)
__device__ __forceinline__ double reciprocal(float s) {
  const double d = s;
  double r = __builtin_amdgcn_rcp(d);
  r = fma(fma(-d, r, 1.0), r, r);
  r = fma(fma(-d, r, 1.0), r, r);
  return s > 0.f ? r : 0.0;
}

// Four values' moments in 8 bits: old codes and scales in, new ones out; mo and vo, the moments in fp32 before they are rounded.
// In 64 bits: which of two codes a value gets does not hang on the order of the operations.  Sixteen lanes have a block.
struct Codes { unsigned m, v; float sm, sv; };
__device__ __forceinline__ Codes quantised_step(const Codes& c, const f32x4& g, const AdamwNow& a, unsigned key, size_t i, f32x4& mo, f32x4& vo) {
  const double b1 = (double)a.beta1 * c.sm, b2 = (double)a.beta2 * c.sv, d1 = 1.0 - (double)a.beta1, d2 = 1.0 - (double)a.beta2;
  double m[4], v[4];
  float tm = 0.f, tv = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int qm = (int)(c.m << (24 - 8 * e)) >> 24, qv = (c.v >> (8 * e)) & 0xff;
    const double gs = (double)g[e] * (double)a.grad_scale;
    m[e] = fma((double)qm, b1, d1 * gs);
    v[e] = fma((double)(qv * qv), b2, d2 * gs * gs);
    mo[e] = (float)m[e];
    vo[e] = (float)v[e];
    // (as whole numbers: NaN is kept)
    tm = __uint_as_float(max(__float_as_uint(tm), __float_as_uint(fabsf(mo[e]))));
    tv = __uint_as_float(max(__float_as_uint(tv), __float_as_uint(vo[e])));
  }
  Codes r;
  r.sm = max16(tm) * (float)(1.0 / 127);
  r.sv = max16(tv) * (float)(1.0 / 65025);
  // a gradient that is not finite: the block's moments are lost, and say so
  if (!(r.sm < INFINITY) || !(r.sv < INFINITY)) r.sm = r.sv = NAN;
  r.m = r.v = 0;
  if (r.sm != r.sm) return r;
  const double im = reciprocal(r.sm), iv = reciprocal(r.sv);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned x = random_bits(i + e, key);
    const float um = ((x & 0xffff) + 0.5f) * (1.f / 65536);    // exact
    const int cm = min(127, max(-127, (int)floor(fma(m[e], im, (double)um))));
    // the code below v: its root in 32 bits, made smaller by more than that can be too large, and one more where that was too much
    const double z = v[e] * iv;
    int q = (int)(__builtin_amdgcn_sqrtf((float)z) * 0.9999995f);
    double rest = z - (double)(q * q);
    const double next = (double)(2 * q + 1);
    if (rest >= next) { ++q; rest -= next; }
    // up where rest > (x >> 16 + 1/2) / 65536 of the step of 2 q + 1, in whole numbers on the right
    int cv = q + (rest * 131072.0 > (double)((2 * (x >> 16) + 1) * (unsigned)(2 * q + 1)) ? 1 : 0);
    cv = min(255, z > 0.0 ? max(1, cv) : cv);
    r.m |= (unsigned)(cm & 0xff) << (8 * e);
    r.v |= (unsigned)cv << (8 * e);
  }
  return r;
}

// A workgroup has 1024 consecutive values, a lane four of them: 16-byte accesses of the fp32 buffers.  Reads and writes 28 bytes a
// value (bf16 gradient and weight), 16.25 with 8-bit moments: bound by memory.  217 M values in 8 bits take 721 us, 4.9 TB/s, 63 M in
// 609 tensors 373 us, 4.7 TB/s; four groups of 1024 a workgroup, loaded ahead, take 14 % longer (more registers, fewer wavefronts).
constexpr unsigned ADAMW_SPAN = 1024;
constexpr unsigned ADAMW_GRID = (1u << 24) - 1;     // workgroups of 256 lanes in a launch, which has less than 2^32
template <bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwSet<EIGHT> u, AdamwNow a) {
  const int tensor = tensor_of(u);
  const AdamwTensor<EIGHT> p = u.t[tensor];
  if (a.live) {
    a.lr = a.live->lr; a.grad_scale = a.live->grad_scale; a.seed = a.live->seed;
    corrections(a, a.live->step ? a.live->step : 1);
  }
  const bool gbf = p.flags & KARMA_ADAMW_GRAD_BF16, obf = p.flags & KARMA_ADAMW_OUT_BF16;
  const uintptr_t odd = (uintptr_t)p.w | (EIGHT ? ((uintptr_t)p.m | (uintptr_t)p.v) * 4 : (uintptr_t)p.m | (uintptr_t)p.v) |
                        (uintptr_t)p.grad * (gbf ? 2 : 1) | (uintptr_t)p.out * (obf ? 2 : 1);
  const size_t i = (size_t)(blockIdx.x - u.first[tensor]) * ADAMW_SPAN + threadIdx.x * 4;
  const bool whole = odd % 16 == 0 && i + 4 <= p.n;
  const f32x4 g = gbf ? load4((const bf16_t*)p.grad, i, p.n, whole) : load4((const float*)p.grad, i, p.n, whole);
  f32x4 w = load4(p.w, i, p.n, whole), m, v;
  if constexpr (EIGHT) {
    const bool some = i / 64 * 64 < p.n;      // the block exists
    const Codes c{load4((const uint8_t*)p.m, i, p.n, whole), load4((const uint8_t*)p.v, i, p.n, whole), some ? p.m_scale[i / 64] : 0.f,
                  some ? p.v_scale[i / 64] : 0.f};
    const Codes r = quantised_step(c, g, a, p.key + a.seed * 0x9e3779b1u, i, m, v);
    store4((uint8_t*)p.m, i, p.n, whole, r.m);
    store4((uint8_t*)p.v, i, p.n, whole, r.v);
    if (threadIdx.x % 16 == 0 && some) { p.m_scale[i / 64] = r.sm; p.v_scale[i / 64] = r.sv; }
  } else {
    m = load4((const float*)p.m, i, p.n, whole);
    v = load4((const float*)p.v, i, p.n, whole);
    const float d1 = (float)(1.0 - (double)a.beta1), d2 = (float)(1.0 - (double)a.beta2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gs = g[e] * a.grad_scale;
      m[e] = a.beta1 * m[e] + d1 * gs;
      v[e] = a.beta2 * v[e] + d2 * gs * gs;
    }
    store4((float*)p.m, i, p.n, whole, m);
    store4((float*)p.v, i, p.n, whole, v);
  }
  // decay and step are added up before the weight sees them: 1 - lr decay in 32 bits is off by a large part of a small decay
  const float shrink = a.lr * p.decay, lr = a.lr * a.c1;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] -= fmaf(shrink, w[e], lr * (m[e] * __builtin_amdgcn_rcpf(sqrtf(v[e]) * a.k2 + a.eps)));
  store4(p.w, i, p.n, whole, w);
  if (p.out) {
    if (obf) store4((bf16_t*)p.out, i, p.n, whole, w);
    else store4((float*)p.out, i, p.n, whole, w);
  }
}

// The moments that 8-bit states stand for: four values a lane; 2.1 bytes in, 8 out (217 M values 365 us, 6.0 TB/s).
struct StatesTensor {
  const uint8_t* m; const uint8_t* v;
  const float* m_scale; const float* v_scale;
  float* m_out; float* v_out;
  size_t n;
};
struct StatesSet {
  static constexpr int MOST = 64;
  StatesTensor t[MOST];
  unsigned first[MOST + 1];
  int n;
};
static_assert(sizeof(StatesSet) <= 4096, "kernel arguments");
__global__ __launch_bounds__(256) void adamw_states_kernel(StatesSet u) {
  const int tensor = tensor_of(u);
  const StatesTensor p = u.t[tensor];
  const uintptr_t odd = ((uintptr_t)p.m | (uintptr_t)p.v) * 4 | (uintptr_t)p.m_out | (uintptr_t)p.v_out;
  const size_t i = (size_t)(blockIdx.x - u.first[tensor]) * ADAMW_SPAN + threadIdx.x * 4;
  if (i >= p.n) return;
  const bool whole = odd % 16 == 0 && i + 4 <= p.n;
  const unsigned cm = load4(p.m, i, p.n, whole), cv = load4(p.v, i, p.n, whole);
  const float sm = p.m_scale[i / 64], sv = p.v_scale[i / 64];
  f32x4 m, v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int q = (cv >> (8 * e)) & 0xff;
    m[e] = (float)((int)(cm << (24 - 8 * e)) >> 24) * sm;
    v[e] = (float)(q * q) * sv;
  }
  store4(p.m_out, i, p.n, whole, m);
  store4(p.v_out, i, p.n, whole, v);
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
bool eight_bits(const karma_adamw_tensor& t) { return t.flags & KARMA_ADAMW_STATES_8BIT; }
bool good_states(const karma_adamw_tensor& t) {
  if (t.n > (uint64_t)ADAMW_GRID * ADAMW_SPAN || (t.flags & ~7u)) return false;
  if (!t.n) return true;
  if (!t.m || !t.v) return false;
  if (eight_bits(t)) return t.m_scale && t.v_scale && aligned_to(t.m_scale, 4) && aligned_to(t.v_scale, 4);
  return aligned_to(t.m, 4) && aligned_to(t.v, 4);
}

// Launches over the tensors of a list for which `fill` fills in a descriptor, as many at a time as the arguments hold.
template <typename Set, typename Fill, typename Launch>
bool in_sets(const karma_adamw_tensor* tensors, uint32_t n, Fill fill, Launch launch) {
  bool launched = false;
  for (uint32_t k = 0; k < n;) {
    Set u;
    u.n = 0;
    u.first[0] = 0;
    uint64_t blocks = 0;
    for (; k < n && u.n < Set::MOST; ++k) {
      const uint64_t more = (tensors[k].n + ADAMW_SPAN - 1) / ADAMW_SPAN;     // (ADAMW_GRID at most)
      if (!more || !fill(u.t[u.n], k)) continue;
      if (blocks + more > ADAMW_GRID) break;
      blocks += more;
      u.first[++u.n] = (unsigned)blocks;
    }
    if (!u.n) continue;
    launch(u, (unsigned)blocks);
    launched = true;
  }
  return launched;
}
template <bool EIGHT>
bool adamw_sets(const karma_adamw_tensor* tensors, uint32_t n, const AdamwNow& a, hipStream_t s) {
  return in_sets<AdamwSet<EIGHT>>(
      tensors, n,
      [&](AdamwTensor<EIGHT>& d, uint32_t k) {
        const karma_adamw_tensor& t = tensors[k];
        if (eight_bits(t) != EIGHT) return false;
        d.w = t.w; d.m = t.m; d.v = t.v; d.grad = t.grad; d.out = t.out; d.n = t.n; d.decay = t.weight_decay; d.flags = t.flags;
        if constexpr (EIGHT) { d.m_scale = t.m_scale; d.v_scale = t.v_scale; d.key = (k + 1) * 0x7f4a7c15u; }
        return true;
      },
      [&](const AdamwSet<EIGHT>& u, unsigned blocks) { hipLaunchKernelGGL(adamw_kernel<EIGHT>, dim3(blocks), dim3(256), 0, s, u, a); });
}

}  // namespace

int adamw(const karma_adamw_tensor* tensors, uint32_t n, const karma_adamw_step& now, const karma_adamw_live* live, hipStream_t s) {
  if (!(now.beta1 >= 0.f && now.beta1 < 1.f && now.beta2 >= 0.f && now.beta2 < 1.f && now.eps >= 0.f) || (!live && !now.step)) return KARMA_E_INVAL;
  if (!aligned_to(live, 4)) return KARMA_E_INVAL;
  for (uint32_t k = 0; k < n; ++k) {
    const karma_adamw_tensor& t = tensors[k];
    if (!good_states(t)) return KARMA_E_INVAL;
    if (t.n && (!t.w || !t.grad || !aligned_to(t.w, 4) || !aligned_to(t.grad, t.flags & KARMA_ADAMW_GRAD_BF16 ? 2 : 4) ||
                !aligned_to(t.out, t.flags & KARMA_ADAMW_OUT_BF16 ? 2 : 4))) return KARMA_E_INVAL;
  }
  AdamwNow a{now.lr, now.beta1, now.beta2, now.eps, now.grad_scale, 0.f, 0.f, now.seed, live};
  if (!live) corrections(a, now.step);
  const bool wide = adamw_sets<false>(tensors, n, a, s), narrow = adamw_sets<true>(tensors, n, a, s);
  return !(wide || narrow) || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int adamw_states(const karma_adamw_tensor* tensors, uint32_t n, float* const* m_out, float* const* v_out, hipStream_t s) {
  for (uint32_t k = 0; k < n; ++k) {
    const karma_adamw_tensor& t = tensors[k];
    if (!eight_bits(t) || !good_states(t)) return KARMA_E_INVAL;
    if (t.n && (!m_out[k] || !v_out[k] || !aligned_to(m_out[k], 4) || !aligned_to(v_out[k], 4))) return KARMA_E_INVAL;
  }
  const bool launched = in_sets<StatesSet>(
      tensors, n,
      [&](StatesTensor& d, uint32_t k) {
        const karma_adamw_tensor& t = tensors[k];
        d = StatesTensor{(const uint8_t*)t.m, (const uint8_t*)t.v, t.m_scale, t.v_scale, m_out[k], v_out[k], (size_t)t.n};
        return true;
      },
      [&](const StatesSet& u, unsigned blocks) { hipLaunchKernelGGL(adamw_states_kernel, dim3(blocks), dim3(256), 0, s, u); });
  return !launched || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

extern "C" int karma_k_adamw(const karma_adamw_tensor* tensors, uint32_t n, const karma_adamw_step* now, const karma_adamw_live* live, void* stream) {
  if (!now || (n && !tensors)) return KARMA_E_INVAL;
  return adamw(tensors, n, *now, live, (hipStream_t)stream);
}
extern "C" int karma_k_adamw_states(const karma_adamw_tensor* tensors, uint32_t n, float* const* m_out, float* const* v_out, void* stream) {
  if (n && (!tensors || !m_out || !v_out)) return KARMA_E_INVAL;
  return adamw_states(tensors, n, m_out, v_out, (hipStream_t)stream);
}
