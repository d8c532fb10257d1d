// AdamW over many tensors at once, moments in fp32 or in 8 bits:
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   w -= lr weight_decay w + lr c1 m / (k2 sqrt(v) + eps),  c1 = 1 / (1 - b1^step),  k2 = 1 / sqrt(1 - b2^step).
// 8 bits: blocks of 64 values share an fp32 scale s.  m = q s with q in -127 .. 127, v = q^2 s with q in 0 .. 255 (the
// square gives small second moments next to large ones four more bits than a linear code).  A value falls between two
// codes and goes to one of them at random, so that its expectation is the value itself: v changes by a thousandth of itself
// a step, and rounding to the nearest code would hold it where it is for good.  The random bits are a hash of the element's
// place and the call's seed.  v > 0 never becomes code 0: m over eps alone would be a huge step.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

constexpr int ADAMW_TENSORS = 44;       // of one launch: their descriptors travel as kernel arguments (4 KB)
constexpr unsigned ADAMW_SPAN = 256;    // values of a workgroup

struct AdamwSet {
  karma_adamw_tensor t[ADAMW_TENSORS];
  unsigned first[ADAMW_TENSORS + 1];    // tensor k has workgroups [first[k], first[k + 1])
  unsigned key[ADAMW_TENSORS];          // of the tensor's random bits, the seed aside
  int n;
};
struct AdamwNow {
  float lr, beta1, beta2, eps, grad_scale;
  unsigned seed;
  unsigned long long step;
  const karma_adamw_live* live;
};
static_assert(sizeof(AdamwSet) + sizeof(AdamwNow) <= 4096, "kernel arguments");

// 1 - beta^step by repeated squaring: one rounding a multiplication, the same on the host and on the device
__host__ __device__ inline double one_minus_power(float beta, unsigned long long step) {
  double p = 1.0, b = beta;
  for (; step; step >>= 1, b *= b)
    if (step & 1) p *= b;
  return 1.0 - p;
}

__device__ __forceinline__ unsigned random_bits(unsigned long long i, unsigned key) {
  unsigned x = (unsigned)i + key;
  x = (x ^ (x >> 16)) * 0x45c3a2adu;
  x = (x ^ (x >> 15)) * 0x2d51f9b5u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float max64(float v) {
  for (int k = 32; k > 0; k >>= 1) {
    const float o = __shfl_xor(v, k);
    v = v != v ? v : (o != o ? o : fmaxf(v, o));    // NaN wins
  }
  return v;
}

__global__ __launch_bounds__(ADAMW_SPAN) void adamw_kernel(AdamwSet u, AdamwNow a) {
  int k = 0;
  while (k + 1 < u.n && blockIdx.x >= u.first[k + 1]) ++k;
  const karma_adamw_tensor& p = u.t[k];
  if (a.live) { a.lr = a.live->lr; a.grad_scale = a.live->grad_scale; a.step = a.live->step ? a.live->step : 1; a.seed = a.live->seed; }
  const float c1 = (float)(1.0 / one_minus_power(a.beta1, a.step)), k2 = (float)(1.0 / sqrt(one_minus_power(a.beta2, a.step)));
  const size_t i = (size_t)(blockIdx.x - u.first[k]) * ADAMW_SPAN + threadIdx.x;
  const bool live = i < p.n, eight = p.flags & KARMA_ADAMW_STATES_8BIT;
  if (!live && !eight) return;
  const float g = !live ? 0.f : (p.flags & KARMA_ADAMW_GRAD_BF16) ? bf2f(((const bf16_t*)p.grad)[i]) : ((const float*)p.grad)[i];
  float m, v;
  if (!eight) {
    const float gs = g * a.grad_scale;
    m = a.beta1 * ((float*)p.m)[i] + (float)(1.0 - (double)a.beta1) * gs;
    v = a.beta2 * ((float*)p.v)[i] + (float)(1.0 - (double)a.beta2) * gs * gs;
    ((float*)p.m)[i] = m;
    ((float*)p.v)[i] = v;
  } else {
#pragma clang fp contract(off)
    const size_t block = i / 64;
    const bool some = block * 64 < p.n;     // the wavefront has a block: block's scales exist
    const int qm = live ? ((const int8_t*)p.m)[i] : 0, qv = live ? ((const uint8_t*)p.v)[i] : 0;
    const double gs = (double)g * (double)a.grad_scale;
    const double md = a.beta1 * (qm * (double)(some ? p.m_scale[block] : 0.f)) + (1.0 - (double)a.beta1) * gs;
    const double vd = a.beta2 * ((double)(qv * qv) * (some ? p.v_scale[block] : 0.f)) + (1.0 - (double)a.beta2) * gs * gs;
    m = (float)md;
    v = (float)vd;
    float sm = max64(live ? fabsf(m) : 0.f) * (float)(1.0 / 127), sv = max64(live ? v : 0.f) * (float)(1.0 / 65025);
    if (!(sm <= 3.4e38f) || !(sv <= 3.4e38f)) sm = sv = NAN;    // a gradient that is not finite: the block's states are lost, and say so
    int cm = 0, cv = 0;
    const unsigned x = random_bits(i, u.key[k] + a.seed * 0x9e3779b1u);
    if (sm > 0.f) cm = min(127, max(-127, (int)floor(md / sm + ((x & 0xffff) + 0.5) / 65536)));
    if (sv > 0.f) {
      const double z = vd / sv, q = fmin(255.0, floor(sqrt(z)));
      cv = min(255, (int)q + (z - q * q > ((x >> 16) + 0.5) / 65536 * (2 * q + 1)));
      if (cv == 0 && z > 0) cv = 1;
    }
    if (some && threadIdx.x % 64 == 0) { p.m_scale[block] = sm; p.v_scale[block] = sv; }
    if (!live) return;
    ((int8_t*)p.m)[i] = (int8_t)cm;
    ((uint8_t*)p.v)[i] = (uint8_t)cv;
  }
  float w = p.w[i];
  w = w - a.lr * p.weight_decay * w - a.lr * (c1 * m / (sqrtf(v) * k2 + a.eps));
  p.w[i] = w;
  if (p.out) {
    if (p.flags & KARMA_ADAMW_OUT_BF16) ((bf16_t*)p.out)[i] = f2bf(w);
    else ((float*)p.out)[i] = w;
  }
}

// the moments that 8-bit states stand for
struct StatesSet {
  const int8_t* m[ADAMW_TENSORS]; const uint8_t* v[ADAMW_TENSORS];
  const float* m_scale[ADAMW_TENSORS]; const float* v_scale[ADAMW_TENSORS];
  float* m_out[ADAMW_TENSORS]; float* v_out[ADAMW_TENSORS];
  unsigned long long size[ADAMW_TENSORS];
  unsigned first[ADAMW_TENSORS + 1];
  int n;
};
static_assert(sizeof(StatesSet) <= 4096, "kernel arguments");
__global__ __launch_bounds__(ADAMW_SPAN) void adamw_states_kernel(StatesSet u) {
  int k = 0;
  while (k + 1 < u.n && blockIdx.x >= u.first[k + 1]) ++k;
  const size_t i = (size_t)(blockIdx.x - u.first[k]) * ADAMW_SPAN + threadIdx.x;
  if (i >= u.size[k]) return;
  const float q = u.v[k][i];
  u.m_out[k][i] = u.m[k][i] * u.m_scale[k][i / 64];
  u.v_out[k][i] = q * q * u.v_scale[k][i / 64];
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
bool eight_bits(const karma_adamw_tensor& t) { return t.flags & KARMA_ADAMW_STATES_8BIT; }
bool good_states(const karma_adamw_tensor& t) {
  if (t.n > ((uint64_t)1 << 40) || (t.flags & ~7u)) return false;
  if (!t.n) return true;
  if (!t.m || !t.v) return false;
  if (eight_bits(t)) return t.m_scale && t.v_scale && aligned_to(t.m_scale, 4) && aligned_to(t.v_scale, 4);
  return aligned_to(t.m, 4) && aligned_to(t.v, 4);
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
  bool launched = false;
  const AdamwNow a{now.lr, now.beta1, now.beta2, now.eps, now.grad_scale, now.seed, now.step, live};
  for (uint32_t k = 0; k < n;) {
    AdamwSet u;
    u.n = 0;
    u.first[0] = 0;
    uint64_t blocks = 0;
    for (; k < n && u.n < ADAMW_TENSORS; ++k) {
      if (!tensors[k].n) continue;
      const uint64_t more = (tensors[k].n + ADAMW_SPAN - 1) / ADAMW_SPAN;
      if (more > INT32_MAX) return KARMA_E_INVAL;
      if (blocks + more > INT32_MAX) break;
      blocks += more;
      u.t[u.n] = tensors[k];
      u.key[u.n] = (k + 1) * 0x7f4a7c15u;
      u.first[++u.n] = (unsigned)blocks;
    }
    if (!u.n) continue;
    hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)blocks), dim3(ADAMW_SPAN), 0, s, u, a);
    launched = true;
  }
  return !launched || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int adamw_states(const karma_adamw_tensor* tensors, uint32_t n, float* const* m_out, float* const* v_out, hipStream_t s) {
  for (uint32_t k = 0; k < n; ++k) {
    const karma_adamw_tensor& t = tensors[k];
    if (!eight_bits(t) || !good_states(t)) return KARMA_E_INVAL;
    if (t.n && (!m_out[k] || !v_out[k] || !aligned_to(m_out[k], 4) || !aligned_to(v_out[k], 4))) return KARMA_E_INVAL;
  }
  bool launched = false;
  for (uint32_t k = 0; k < n;) {
    StatesSet u;
    u.n = 0;
    u.first[0] = 0;
    uint64_t blocks = 0;
    for (; k < n && u.n < ADAMW_TENSORS; ++k) {
      const karma_adamw_tensor& t = tensors[k];
      if (!t.n) continue;
      const uint64_t more = (t.n + ADAMW_SPAN - 1) / ADAMW_SPAN;
      if (more > INT32_MAX) return KARMA_E_INVAL;
      if (blocks + more > INT32_MAX) break;
      blocks += more;
      u.m[u.n] = (const int8_t*)t.m; u.v[u.n] = (const uint8_t*)t.v; u.m_scale[u.n] = t.m_scale; u.v_scale[u.n] = t.v_scale;
      u.m_out[u.n] = m_out[k]; u.v_out[u.n] = v_out[k]; u.size[u.n] = t.n;
      u.first[++u.n] = (unsigned)blocks;
    }
    if (!u.n) continue;
    hipLaunchKernelGGL(adamw_states_kernel, dim3((unsigned)blocks), dim3(ADAMW_SPAN), 0, s, u);
    launched = true;
  }
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
